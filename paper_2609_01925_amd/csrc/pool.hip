// Bookkeeping of a paged cache's pages on the device: which are in use and how often, and the
// tables that sequences find theirs in.  Nothing here reads K or V; one pool serves the caches
// of all layers, and the page copies that a fork or a compaction asks for come out as pairs.
//
// pool = uses of each page [n_pages] (int32), then one bit a page that is in use (32 a word,
// lowest page first).  The bits are what a search for free pages reads: 4 KB for 32768 pages.
//
// All of it is latency: a few kilobytes behind chains of dependent loads.  What has to be in
// order (who is served, with which page) is worked out by one workgroup with scans, so that the same
// calls always give the same pages, lowest first; atomics only add, subtract and set bits.  Measured, us: a reservation for 64 of
// 256 sequences from 32768 pages 14.4, the free before it 7.7; 24 forks 8.3 and the free before them 3.1; the compaction of 4096
// pages 4.4 and its tables' 4.9.
#include "cache_device.h"

namespace crisp {

namespace {

constexpr int kThreads = 1024;
constexpr int kWavesPool = kThreads / kWave;
constexpr int kBuf = 4096;  // free pages collected at a time
// Up to so many row entries a fork fills the new rows in its own launch.  A free and a fork of 16, in a second launch / here,
// us, called from a host program and replayed from a graph: 64 slots 18.1 / 15.2 and 11.1 / 9.9; 256 (the limit) 18.0 / 15.1 and
// 11.6 / 13.3; 512 18.1 / 17.0 and 12.8 / 16.7; 1024 18.0 / 27.1 and 15.0 / 26.6.  The limit is where a program that calls gains still; a
// replayed graph, whose launches cost less, gains up to about half of it and loses up to 1.7 us there.
constexpr int64_t kShareHere = 4096;
constexpr int kPerThread = kPoolMaxSeqs / kThreads;
constexpr int kMostFree = 1 << 16;  // workgroups of a free; each takes every so-many-th sequence
static_assert(kPoolMaxSeqs <= kBuf, "a fork collects its pages at once");

__device__ __forceinline__ uint32_t* bits_of(int32_t* pool, int n_pages) { return reinterpret_cast<uint32_t*>(pool + n_pages); }
__device__ __forceinline__ uint32_t load_word(const uint32_t* p) {  // past L1: other threads set bits atomically
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// The pages of word i that exist.
__device__ __forceinline__ uint32_t word_mask(int i, int n_pages) {
  const int left = n_pages - 32 * i;
  return left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1u;
}

struct PoolLds {
  int wsum[kWavesPool];
  int buf[kBuf];
};

// Pages not in use, lowest first, into buf from word *word on until `want` (<= kBuf) are found; returns
// the number found (it may pass `want`, of which no more than kBuf are in buf).  *word is then where
// to look on: the words before it hold none but those in buf.
__device__ __forceinline__ int collect_free(const uint32_t* bits, int n_pages, int want, int* word, PoolLds& l) {
  const int words = (n_pages + 31) / 32;
  int found = 0;
  while (found < want && *word < words) {
    const int i = *word + (int)threadIdx.x;
    uint32_t f = i < words ? ~load_word(bits + i) & word_mask(i, n_pages) : 0u;
    const int cnt = __popc(f);
    int total;
    __syncthreads();
    int at = found + block_scan<int, kWavesPool>(cnt, l.wsum, &total) - cnt;
    for (; f && at < want; f &= f - 1, ++at) l.buf[at] = 32 * i + __builtin_ctz(f);
    found += total;
    if (found <= want) *word += kThreads;
  }
  __syncthreads();
  return found;
}

// Marks the n lowest free pages as in use, n of them being free: a word a thread, so that no two
// threads write one.
__device__ __forceinline__ void take_lowest(uint32_t* bits, int n_pages, int n, PoolLds& l) {
  const int words = (n_pages + 31) / 32;
  int found = 0;
  for (int w0 = 0; w0 < words && found < n; w0 += kThreads) {
    const int i = w0 + (int)threadIdx.x;
    const uint32_t was = i < words ? load_word(bits + i) : ~0u;
    uint32_t f = ~was & word_mask(i, n_pages);
    const int cnt = __popc(f);
    int total;
    __syncthreads();
    const int at = found + block_scan<int, kWavesPool>(cnt, l.wsum, &total) - cnt;
    uint32_t left = f;  // what stays free: all but the lowest n - at
    if (at + cnt <= n) left = 0;
    else
      for (int k = at; k < n; ++k) left &= left - 1;
    if (f != left) bits[i] = was | (f & ~left);
    found += total;
  }
}

// Pages not in use among the words from `word` on, counted by the workgroup.
__device__ __forceinline__ int count_free(const uint32_t* bits, int n_pages, int word, int* wsum) {
  const int words = (n_pages + 31) / 32;
  int n = 0;
#pragma unroll 4
  for (int i = word + (int)threadIdx.x; i < words; i += kThreads) n += __popc(~load_word(bits + i) & word_mask(i, n_pages));
  int total;
  __syncthreads();
  block_scan<int, kWavesPool>(n, wsum, &total);
  return total;
}

__device__ __forceinline__ void take_page(int32_t* pool, uint32_t* bits, int page) {
  pool[page] = 1;
  atomicOr(bits + (page >> 5), 1u << (page & 31));
}

__global__ __launch_bounds__(256) void pool_init(int32_t* pool, int64_t words) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < words) pool[i] = 0;
}

// Sequence s asks for room for counts[s] tokens behind its seq_len[s]: the slots len / B ..
// ceil((len + count) / B) - 1 that hold no page.  Asked for in order of sequence and slot; a
// sequence whose running sum (its own included) passes the free pages, whose slots pass the
// table, or one of whose slots has a page that is used more than once (tokens were taken back into
// what a fork shares: rows written there would change the other's) gets none.  The slots of all sequences in a row are looked at kEach a thread; where one
// round covers them all, what was read serves for the assignment too.
__global__ __launch_bounds__(kThreads) void pool_reserve(int n_pages, int B, int n_seqs, int max_pages, int32_t* pool,
                                                         int32_t* table, const int32_t* seq_len, const int32_t* counts,
                                                         int32_t* granted) {
  constexpr int kEach = 4, kRound = kEach * kThreads;
  __shared__ PoolLds l;
  constexpr int kShared = 1 << 30;
  // place of a sequence's first slot among all, what leads from a place to its table entry, and
  // its missing pages and kShared if one is shared (then: whether it is served)
  __shared__ int first[kPoolMaxSeqs + 1], entry[kPoolMaxSeqs], miss[kPoolMaxSeqs];
  uint32_t* bits = bits_of(pool, n_pages);
  const int tid = threadIdx.x;
  const int per = (n_seqs + kThreads - 1) / kThreads;
  bool fits[kPerThread];
  int ask[kPerThread], range[kPerThread], from[kPerThread], own = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int s = tid * per + i;
    range[i] = 0, fits[i] = false, ask[i] = 0, from[i] = 0;
    if (i < per && s < n_seqs) {
      const int len = (int)min((int64_t)max(seq_len[s], 0), (int64_t)max_pages * B);
      ask[i] = max(counts[s], 0);
      const int64_t last = ((int64_t)len + ask[i] + B - 1) / B;
      fits[i] = ask[i] > 0 && last <= max_pages;
      from[i] = len / B;
      if (fits[i]) range[i] = (int)last - from[i];
    }
    own += range[i];
  }
  int total;
  int at = block_scan<int, kWavesPool>(own, l.wsum, &total) - own;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int s = tid * per + i;
    if (i < per && s < n_seqs) {
      first[s] = at;
      entry[s] = s * max_pages + from[i] - at;  // fits: the table has less than 2^31 entries
      miss[s] = 0;
      at += range[i];
    }
  }
  if (tid == 0) first[n_seqs] = total;
  // the lowest free pages, and how many there are
  int word = 0;
  int n_free = collect_free(bits, n_pages, kBuf, &word, l);  // its barriers also publish first, entry and miss
  if (n_free > kBuf) {  // those of the words up to the last one looked at are in n_free
    n_free += count_free(bits, n_pages, word + kThreads, l.wsum);
  } else if (n_free == kBuf) {
    n_free += count_free(bits, n_pages, word, l.wsum);
  }
  struct Slots {
    int s[kEach], e[kEach], page[kEach];
    bool lack[kEach];
  };
  const auto read = [&](int p0, Slots& x) {
    const int p = p0 + kEach * tid;
    int lo = 0, hi = n_seqs;  // first[lo] <= p < first[hi]
    if (p < total)
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first[mid] <= p) lo = mid;
        else hi = mid;
      }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      x.lack[k] = false;
      x.page[k] = -1;
      if (p + k < total) {
        while (first[lo + 1] <= p + k) ++lo;  // ends: first[n_seqs] = total
        x.s[k] = lo;
        x.e[k] = entry[lo] + p + k;
        x.page[k] = table[x.e[k]];
        x.lack[k] = x.page[k] < 0;
      }
    }
  };
  Slots x;
  for (int64_t p0 = 0; p0 < total; p0 += kRound) {  // 64 bits: total may be 2^31 - 1
    read((int)p0, x);
    int n = 0;  // missing pages of one sequence among the thread's slots
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      n += x.lack[k];
      if (n && (k == kEach - 1 || !x.lack[k + 1] || x.s[k + 1] != x.s[k])) {
        atomicAdd(&miss[x.s[k]], n);
        n = 0;
      }
      if (x.page[k] >= 0 && x.page[k] < n_pages && pool[x.page[k]] > 1) atomicOr(&miss[x.s[k]], kShared);
    }
  }
  __syncthreads();
  own = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i)
    if (i < per && tid * per + i < n_seqs) {
      const int m = miss[tid * per + i];
      if (m & kShared) {
        fits[i] = false;
        miss[tid * per + i] = 0;
      } else {
        own += m;
      }
    }
  int all;
  int sum = block_scan<int, kWavesPool>(own, l.wsum, &all) - own;
  int taken = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int s = tid * per + i;
    if (i >= per || s >= n_seqs) break;
    const int m = miss[s];
    sum += m;
    const bool ok = fits[i] && (m == 0 || sum <= n_free);
    granted[s] = ok ? ask[i] : 0;
    miss[s] = ok;
    if (ok) taken += m;
  }
  __syncthreads();
  int want;
  block_scan<int, kWavesPool>(taken, l.wsum, &want);
  for (int done = 0; done < want; done += kBuf) {
    const int now = min(want - done, kBuf);
    if (done > 0) {
      word = 0;
      collect_free(bits, n_pages, now, &word, l);
    }
    int rank = 0;
    for (int64_t p0 = 0; p0 < total && rank < now; p0 += kRound) {
      if (total > kRound) read((int)p0, x);  // otherwise x is still that of the only round
      int mine = 0;
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        x.lack[k] = x.lack[k] && miss[x.s[k]] && (done == 0 || table[x.e[k]] < 0);
        mine += x.lack[k];
      }
      int here;
      __syncthreads();
      int k0 = rank + block_scan<int, kWavesPool>(mine, l.wsum, &here) - mine;
#pragma unroll
      for (int k = 0; k < kEach; ++k)
        if (x.lack[k]) {
          if (k0 < now) {
            table[x.e[k]] = l.buf[k0];
            pool[l.buf[k0]] = 1;
          }
          ++k0;
        }
      rank += here;
    }
    take_lowest(bits, n_pages, now, l);
    __threadfence();  // the next round looks for free pages in what this one has set
    __syncthreads();
  }
}

// Slot j of a fork that holds len tokens: a full page is listed in the new row and counted once more, the
// slots behind the last page are empty (the partial page's slot is set already).
__device__ __forceinline__ void share_slot(int n_pages, int B, int32_t* pool, const int32_t* from, int32_t* to, int len, int j) {
  if (j < len / B) {
    const int p = from[j];
    to[j] = p;
    if (p >= 0 && p < n_pages) atomicAdd(pool + p, 1);
  } else if (j >= (len + B - 1) / B) {
    to[j] = -1;
  }
}

// Fork i makes the empty sequence dst[i] hold what src[i] holds.  Of two forks into one sequence
// the first counts.  A partial last page is not shared but copied to the lowest free page:
// copies[i] = (page, its copy), (-1, -1) where there is nothing to copy, (-2, -2) where the fork
// is refused.  Lengths are those before the call.  share: the rows are filled here too.
__global__ __launch_bounds__(kThreads) void pool_fork(int n_pages, int B, int n_seqs, int max_pages, int32_t* pool,
                                                      int32_t* table, int32_t* seq_len, const int32_t* src,
                                                      const int32_t* dst, int n, int32_t* copies,
                                                      bool share) {
  __shared__ PoolLds l;
  __shared__ int lens[kPoolMaxSeqs], owner[kPoolMaxSeqs];
  uint32_t* bits = bits_of(pool, n_pages);
  const int tid = threadIdx.x;
  const int per = (n + kThreads - 1) / kThreads;
  for (int i = tid; i < n_seqs; i += kThreads) owner[i] = n;
  for (int i = tid; i < n; i += kThreads) {
    const int s = src[i], d = dst[i];
    int len = -1;
    if (s >= 0 && s < n_seqs && d >= 0 && d < n_seqs && s != d && seq_len[d] == 0 &&
        (max_pages == 0 || table[(int64_t)d * max_pages] < 0))
      len = (int)min((int64_t)max(seq_len[s], 0), (int64_t)max_pages * B);
    lens[i] = len;
  }
  __syncthreads();
  for (int i = tid; i < n; i += kThreads)
    if (lens[i] >= 0) atomicMin(&owner[dst[i]], i);
  __syncthreads();
  bool ok[kPerThread];
  int tail[kPerThread], own = 0;
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    ok[k] = i < n && lens[i] >= 0 && owner[dst[i]] == i;
    tail[k] = -1;
    if (ok[k] && lens[i] % B) {
      tail[k] = table[(int64_t)src[i] * max_pages + lens[i] / B];
      ok[k] = tail[k] >= 0 && tail[k] < n_pages;
      own += ok[k];
    }
  }
  int need;
  int rank = block_scan<int, kWavesPool>(own, l.wsum, &need) - own;
  int word = 0;
  const int n_free = collect_free(bits, n_pages, need, &word, l);  // need <= kPoolMaxSeqs <= kBuf
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    if (i >= n) break;
    int from = -2, to = -2;
    if (ok[k]) {
      const bool copy = lens[i] % B != 0;
      const int mine = copy ? rank++ : 0;
      if (!copy || mine < n_free) {
        from = to = -1;
        if (copy) {
          from = tail[k];
          to = l.buf[mine];
          table[(int64_t)dst[i] * max_pages + lens[i] / B] = to;
          take_page(pool, bits, to);
        }
        seq_len[dst[i]] = lens[i];
      }
    }
    if (from == -2) lens[i] = -1;
    copies[2 * i] = from;
    copies[2 * i + 1] = to;
  }
  if (!share) return;
  __syncthreads();
  for (int e = tid; e < n * max_pages; e += kThreads) {
    const int i = e / max_pages, j = e % max_pages;
    if (lens[i] >= 0)
      share_slot(n_pages, B, pool, table + (int64_t)src[i] * max_pages, table + (int64_t)dst[i] * max_pages, lens[i], j);
  }
}

// The rows of the granted forks, a workgroup each.
__global__ __launch_bounds__(256) void pool_share(int n_pages, int B, int max_pages, int32_t* pool, int32_t* table,
                                                  const int32_t* seq_len, const int32_t* src, const int32_t* dst,
                                                  const int32_t* copies) {
  const int i = blockIdx.x;
  if (copies[2 * i] == -2) return;
  for (int j = threadIdx.x; j < max_pages; j += 256)
    share_slot(n_pages, B, pool, table + (int64_t)src[i] * max_pages, table + (int64_t)dst[i] * max_pages, seq_len[dst[i]], j);
}

// Every page in the row of a freed sequence loses one use.  The exchange gives each page to one
// thread, also where a sequence is listed twice.
__global__ __launch_bounds__(256) void pool_free(int n_pages, int n_seqs, int max_pages, int32_t* pool, int32_t* table,
                                                 int32_t* seq_len, const int32_t* ids, int n) {
  uint32_t* bits = bits_of(pool, n_pages);
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const int s = ids[i];
    if (s < 0 || s >= n_seqs) continue;
    int32_t* row = table + (int64_t)s * max_pages;
    for (int j = threadIdx.x; j < max_pages; j += 256) {
      const int p = atomicExch(row + j, -1);
      if (p < 0 || p >= n_pages) continue;
      const int before = atomicSub(pool + p, 1);
      if (before == 1) atomicAnd(bits + (p >> 5), ~(1u << (p & 31)));
      if (before <= 0) atomicAdd(pool + p, 1);  // not in use: nothing to take away
    }
    if (threadIdx.x == 0) seq_len[s] = 0;
  }
}

// With U pages in use, the k-th free page below U takes the k-th page in use from U on.  Sources and
// destinations are apart, so the copies may run in any order.
__global__ __launch_bounds__(kThreads) void pool_compact(int n_pages, int32_t* pool, int32_t* moves, int32_t* count) {
  __shared__ int wsum[kWavesPool];
  uint32_t* bits = bits_of(pool, n_pages);
  const int tid = threadIdx.x;
  const int words = (n_pages + 31) / 32;
  const int used = n_pages - count_free(bits, n_pages, 0, wsum);
  int holes = 0, movers = 0;
  for (int w0 = 0; w0 < words; w0 += kThreads) {
    const int i = w0 + tid;
    const uint32_t in = i < words ? bits[i] & word_mask(i, n_pages) : 0u;
    const uint32_t front = i < words ? word_mask(i, used) : 0u;  // pages below U
    uint32_t hole = ~in & front, mover = in & ~front;
    const int nh = __popc(hole), nm = __popc(mover);
    int total;
    __syncthreads();
    int at = holes + block_scan<int, kWavesPool>(nh, wsum, &total) - nh;
    holes += total;
    for (; hole; hole &= hole - 1, ++at) moves[2 * at + 1] = 32 * i + __builtin_ctz(hole);
    __syncthreads();
    at = movers + block_scan<int, kWavesPool>(nm, wsum, &total) - nm;
    movers += total;
    for (; mover; mover &= mover - 1, ++at) moves[2 * at] = 32 * i + __builtin_ctz(mover);
  }
  __syncthreads();
  for (int k = tid; k < holes; k += kThreads) {
    const int from = moves[2 * k], to = moves[2 * k + 1];
    pool[to] = pool[from];
    pool[from] = 0;
  }
  for (int i = tid; i < words; i += kThreads) bits[i] = word_mask(i, used);
  if (tid == 0) *count = holes;
}

// The tables' entries follow the moves (ascending in their source); the pairs behind the last are -1.
__global__ __launch_bounds__(256) void pool_retable(int64_t entries, int cap, int32_t* table, int32_t* moves,
                                                    const int32_t* count) {
  const int n = *count;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < entries + cap; x += (int64_t)gridDim.x * 256) {
    if (x >= entries) {
      const int k = (int)(x - entries);
      if (k >= n) moves[2 * k] = moves[2 * k + 1] = -1;
      continue;
    }
    if (n == 0) continue;
    const int p = table[x];
    if (p < moves[0]) continue;
    int lo = 0, hi = n;  // moves[2 lo] <= p < moves[2 hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (moves[2 * mid] <= p) lo = mid;
      else hi = mid;
    }
    if (moves[2 * lo] == p) table[x] = moves[2 * lo + 1];
  }
}

}  // namespace

hipError_t launch_pool_init(int n_pages, int32_t* pool, hipStream_t stream) {
  const int64_t words = pool_words(n_pages);
  hipLaunchKernelGGL(pool_init, dim3((unsigned)((words + 255) / 256)), dim3(256), 0, stream, pool, words);
  return hipGetLastError();
}

hipError_t launch_pool_reserve(int n_pages, int block, int n_seqs, int max_pages, int32_t* pool, int32_t* table,
                               const int32_t* seq_len, const int32_t* counts, int32_t* granted, hipStream_t stream) {
  hipLaunchKernelGGL(pool_reserve, dim3(1), dim3(kThreads), 0, stream, n_pages, block, n_seqs, max_pages, pool, table,
                     seq_len, counts, granted);
  return hipGetLastError();
}

hipError_t launch_pool_fork(int n_pages, int block, int n_seqs, int max_pages, int32_t* pool, int32_t* table,
                            int32_t* seq_len, const int32_t* src, const int32_t* dst, int n, int32_t* copies,
                            hipStream_t stream) {
  const bool share = (int64_t)n * max_pages <= kShareHere;
  hipLaunchKernelGGL(pool_fork, dim3(1), dim3(kThreads), 0, stream, n_pages, block, n_seqs, max_pages, pool, table,
                     seq_len, src, dst, n, copies, share);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || share) return e;
  hipLaunchKernelGGL(pool_share, dim3((unsigned)n), dim3(256), 0, stream, n_pages, block, max_pages, pool, table,
                     (const int32_t*)seq_len, src, dst, (const int32_t*)copies);
  return hipGetLastError();
}

hipError_t launch_pool_free(int n_pages, int n_seqs, int max_pages, int32_t* pool, int32_t* table, int32_t* seq_len,
                            const int32_t* ids, int n, hipStream_t stream) {
  hipLaunchKernelGGL(pool_free, dim3((unsigned)(n < kMostFree ? n : kMostFree)), dim3(256), 0, stream, n_pages, n_seqs,
                     max_pages, pool, table, seq_len, ids, n);
  return hipGetLastError();
}

hipError_t launch_pool_compact(int n_pages, int n_seqs, int max_pages, int32_t* pool, int32_t* table, int32_t* moves,
                               int32_t* count, hipStream_t stream) {
  hipLaunchKernelGGL(pool_compact, dim3(1), dim3(kThreads), 0, stream, n_pages, pool, moves, count);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int cap = n_pages / 2 > 1 ? n_pages / 2 : 1;
  const int64_t entries = (int64_t)n_seqs * max_pages, blocks = (entries + cap + 255) / 256;
  hipLaunchKernelGGL(pool_retable, dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(256), 0, stream, entries, cap,
                     table, moves, (const int32_t*)count);
  return hipGetLastError();
}

}  // namespace crisp
