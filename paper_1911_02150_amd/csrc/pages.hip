// Who holds which page of a pool.  refs[page]: how many entries of tables name it; a page with none (or fewer) is free.  Pages are given out from the lowest
// free one on, so that what a call does depends on its arguments alone.
#include "paged.hpp"

namespace mqa {
namespace {

__device__ __forceinline__ bool is_page(int entry, int num_pages) { return (unsigned)entry < (unsigned)num_pages; }
__device__ __forceinline__ int pages_of(int len, int page_size) { return (int)(((unsigned)len + (unsigned)page_size - 1) / (unsigned)page_size); }

// ---------------------------------------------------------------- fork, free
// A thread has a column of kRun neighbouring sequences' entries, and one atomic for those that follow each other and name the same page, as siblings' do: the counts' atomics bound it, and for
// few entries the launch and three reads in a row (one of 256 pages to 512: 5.6 us, an entry a thread 11.9, runs of eight 5.3; 64 to 512 of them 3.6, 3.1 and 4.5).
constexpr int kRun = 4;

template <int SIGN>
struct Run {                             // of one page's entries
  int page = -1, count = 0;
  __device__ __forceinline__ void end(int32_t* refs) {
    if (count) atomicAdd(refs + page, SIGN * count);
  }
  __device__ __forceinline__ void add(int32_t* refs, int entry) {
    if (entry != page) {
      end(refs);
      page = entry;
      count = 0;
    }
    ++count;
  }
};

__global__ __launch_bounds__(256)
void fork_kernel(PageFork p) {
  const unsigned idx = blockIdx.x * 256u + threadIdx.x;
  const int j0 = kRun * (int)(idx / (unsigned)p.max_pages), x = (int)(idx % (unsigned)p.max_pages);
  if (j0 >= p.b_out) return;
  int parent[kRun], entry[kRun], len[kRun];
#pragma unroll
  for (int u = 0; u < kRun; ++u) parent[u] = p.parents[min(j0 + u, p.b_out - 1)];
#pragma unroll
  for (int u = 0; u < kRun; ++u) {
    const bool there = (unsigned)parent[u] < (unsigned)p.b_in;
    entry[u] = there ? p.table_in[(size_t)parent[u] * p.max_pages + x] : -1;
    len[u] = there ? p.lens_in[parent[u]] : 0;
  }
  Run<1> run;
#pragma unroll
  for (int u = 0; u < kRun; ++u) {
    if (j0 + u >= p.b_out) break;
    len[u] = min(max(len[u], 0), p.max_pages * p.page_size);
    if (x >= pages_of(len[u], p.page_size) || !is_page(entry[u], p.num_pages)) entry[u] = -1;
    if (entry[u] >= 0) run.add(p.refs, entry[u]);
    p.table_out[(size_t)(j0 + u) * p.max_pages + x] = entry[u];
    if (x == 0) p.lens_out[j0 + u] = len[u];
  }
  run.end(p.refs);
}

__global__ __launch_bounds__(256)
void free_kernel(PageFree p) {
  const unsigned idx = blockIdx.x * 256u + threadIdx.x;
  const int i0 = kRun * (int)(idx / (unsigned)p.max_pages), x = (int)(idx % (unsigned)p.max_pages);
  if (i0 >= p.b) return;
  int entry[kRun], len[kRun];
#pragma unroll
  for (int u = 0; u < kRun; ++u) {
    const int i = min(i0 + u, p.b - 1);
    entry[u] = p.table[(size_t)i * p.max_pages + x];
    len[u] = p.lens[i];
  }
  Run<-1> run;
#pragma unroll
  for (int u = 0; u < kRun; ++u) {
    if (i0 + u >= p.b) break;
    if (x < pages_of(min(max(len[u], 0), p.max_pages * p.page_size), p.page_size)) continue;
    if (is_page(entry[u], p.num_pages)) run.add(p.refs, entry[u]);
    if (entry[u] != -1) p.table[(size_t)(i0 + u) * p.max_pages + x] = -1;
  }
  run.end(p.refs);
}

// ---------------------------------------------------------------- sums over a workgroup
template <int THREADS>
__device__ __forceinline__ int before_me(int x, int* s_waves, int* all) {      // (s_waves is the call's own until the second barrier after it)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(incl, off);
    if (lane >= off) incl += y;
  }
  if (lane == 63) s_waves[wave] = incl;
  __syncthreads();
  int before = incl - x, sum = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) before += s_waves[w];
    sum += s_waves[w];
  }
  *all = sum;
  return before;
}

// Which of the eight pages from `first` (a multiple of 8) on have a count above 0, and which are there at all.
__device__ __forceinline__ uint32_t in_use8(const int32_t* refs, int first, int num_pages) {
  uint32_t bits = 0;
  if (first + 8 <= num_pages) {
    const int4 a = reinterpret_cast<const int4*>(refs + first)[0], b = reinterpret_cast<const int4*>(refs + first)[1];
    bits = (a.x > 0) | (a.y > 0) << 1 | (a.z > 0) << 2 | (a.w > 0) << 3 | (b.x > 0) << 4 | (b.y > 0) << 5 | (b.z > 0) << 6 | (b.w > 0) << 7;
  } else {
    for (int x = 0; first + x < num_pages; ++x) bits |= (uint32_t)(refs[first + x] > 0) << x;
  }
  return bits;
}
__device__ __forceinline__ uint32_t there8(int first, int num_pages) { return first >= num_pages ? 0u : first + 8 <= num_pages ? 0xffu : (1u << (num_pages - first)) - 1; }

// ---------------------------------------------------------------- reserve
// One workgroup, in steps:
//  1. of every page that sequences are about to write behind rows that others share: how many are, and the last of them
//  2. what every sequence needs: per page of its new positions nothing (kKept), a page (kMissing), or a page in place of a shared one (that one's number);
//     and how many pages that makes, running over the sequences (a thread has four neighbouring entries at a time)
//  3. as many free pages as are needed, or as there are
//  4. to the sequences whose running number is there: their pages
// (Step 4 reads what step 2 has written down and no counts, since it changes them.)
// What bounds it is the latency of what a step reads, a round of 4096 entries after the other (a prompt of 4096 in pages of 16 8 us; 64 of 512 10.1; with a sequence's entries one thread's 106 and 25.6).
constexpr int kReserveThreads = 1024;
constexpr int kKept = -2, kMissing = -1;

struct ReserveSpace {
  int2* writers;       // [num_pages]: how many, the last (written before they are read, where they are read)
  int2* needs;         // [b, slots]: what, and which of the pages it would be
  int2* running;       // [b]: pages before the sequence (-1: it keeps one that others are about to leave), and with it
  int32_t* pages;      // free ones
  int slots;
  size_t bytes;
};
__host__ __device__ ReserveSpace reserve_space(int b, int n, int num_pages, int page_size, void* at) {
  ReserveSpace s;
  s.slots = (int)((n + (long long)page_size - 2) / page_size) + 1;      // pages that n rows reach, at most
  const size_t writers = ((size_t)num_pages * 8 + 15) & ~(size_t)15, needs = ((size_t)b * s.slots * 8 + 15) & ~(size_t)15, running = ((size_t)b * 8 + 15) & ~(size_t)15;
  unsigned char* const p = static_cast<unsigned char*>(at);
  s.writers = reinterpret_cast<int2*>(p);
  s.needs = reinterpret_cast<int2*>(p + writers);
  s.running = reinterpret_cast<int2*>(p + writers + needs);
  s.pages = reinterpret_cast<int32_t*>(p + writers + needs + running);
  s.bytes = writers + needs + running + (((size_t)num_pages * 4 + 15) & ~(size_t)15);
  return s;
}

// put(x, page) for the x-th free page, x < total at least if there are so many; how many it has come to.  `used`: of a thread's first eight pages.
template <int T, typename Put>
__device__ __forceinline__ int find_free(const int32_t* refs, int num_pages, uint32_t used, int total, int* s_waves, Put put) {
  const int tid = threadIdx.x;
  auto give = [&](uint32_t free, int first, int at) {
    for (; free; free &= free - 1) put(at++, first + __ffs(free) - 1);
  };
  if (total == 0) return 0;
  uint32_t free = ~used & there8(8 * tid, num_pages);
  int found, at = before_me<T>(__popc(free), s_waves, &found);
  give(free, 8 * tid, at);
  for (int base = 8 * T; base < num_pages && found < total; base += 16 * T) {      // then twice eight
    uint32_t more[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) more[g] = ~in_use8(refs, base + 8 * (T * g + tid), num_pages) & there8(base + 8 * (T * g + tid), num_pages);
    __syncthreads();
    int all;
    const int before = before_me<T>(__popc(more[0]) | __popc(more[1]) << 16, s_waves, &all);      // (up to 8 T each)
    give(more[0], base + 8 * tid, found + (before & 0xffff));
    found += all & 0xffff;
    give(more[1], base + 8 * (T + tid), found + (before >> 16));
    found += all >> 16;
  }
  return found;
}

// The new positions of sequence i: false: there are none, or no room.
struct Wanted { int len, count, first, last; bool begun; };      // pages first .. last - 1; the first one has rows already
__device__ __forceinline__ bool wanted(const PageReserve& p, int i, Wanted* w) {
  w->len = p.lens[i];
  w->count = p.counts ? min(max(p.counts[i], 0), p.n) : p.n;
  if (w->len < 0 || w->len > p.max_pages * p.page_size - w->count || w->count == 0) return false;
  w->first = w->len / p.page_size;
  w->last = pages_of(w->len + w->count, p.page_size);
  w->begun = w->len - w->first * p.page_size != 0;
  return true;
}

__global__ __launch_bounds__(kReserveThreads)
void reserve_kernel(PageReserve p, void* workspace) {
  __shared__ int s_waves[2][kReserveThreads / 64];
  const int tid = threadIdx.x;
  const ReserveSpace s = reserve_space(p.b, p.n, p.num_pages, p.page_size, workspace);
  Wanted w;
  auto begun_page = [&](int i) {       // the shared page that sequence i writes to behind its rows, or -1
    if (!wanted(p, i, &w) || !w.begun) return -1;
    const int entry = p.table[(size_t)i * p.max_pages + w.first];
    return is_page(entry, p.num_pages) && p.refs[entry] > 1 ? entry : -1;
  };
  uint32_t used = in_use8(p.refs, 8 * tid, p.num_pages);      // (for step 3, its first pages)
  int mine = 0;
  for (int i = tid; i < p.b; i += kReserveThreads) {
    const int page = begun_page(i);
    s.running[i].x = page;
    if (page >= 0) {
      s.writers[page] = make_int2(0, -1);
      mine = 1;
    }
  }
  __threadfence_block();
  if (__syncthreads_or(mine)) {
    for (int i = tid; i < p.b; i += kReserveThreads) {
      const int page = s.running[i].x;
      if (page >= 0) {
        atomicAdd(&s.writers[page].x, 1);
        atomicMax(&s.writers[page].y, i);
      }
    }
    __threadfence_block();
    __syncthreads();
  }
  const int items = p.b * s.slots;
  int total = 0;
  for (int base = 0, turn = 0; base < items; base += 4 * kReserveThreads, turn ^= 1) {
    int seq[4], slot[4], entry[4], refs[4], need[4], needs = 0;
    bool ours[4], begun[4], keeps[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int item = min(base + 4 * tid + u, items - 1);
      seq[u] = item / s.slots;
      slot[u] = item - seq[u] * s.slots;
      ours[u] = wanted(p, seq[u], &w) && w.first + slot[u] < w.last && base + 4 * tid + u < items;
      begun[u] = w.begun && slot[u] == 0;
      entry[u] = ours[u] ? p.table[(size_t)seq[u] * p.max_pages + w.first + slot[u]] : -1;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) refs[u] = is_page(entry[u], p.num_pages) ? p.refs[entry[u]] : 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool there = is_page(entry[u], p.num_pages);
      need[u] = !ours[u] || (there && refs[u] <= 1) ? kKept : there ? entry[u] : kMissing;
      keeps[u] = false;
      if (ours[u] && begun[u]) {
        if (!there) need[u] = kKept;                   // (rows on no page: they stay nowhere)
        if (need[u] >= 0) {
          // (past L1, which the atomics do not go through)
          const int others = __hip_atomic_load(&s.writers[entry[u]].x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          if (others == refs[u] && __hip_atomic_load(&s.writers[entry[u]].y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == seq[u]) { need[u] = kKept; keeps[u] = true; }
        }
      }
      needs += need[u] != kKept;
    }
    int all, before = total + before_me<kReserveThreads>(needs, s_waves[turn], &all);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (base + 4 * tid + u >= items) break;
      s.needs[base + 4 * tid + u] = make_int2(need[u], before);
      // (who keeps a page that others are about to leave may do so only if they do)
      if (slot[u] == 0) s.running[seq[u]].x = keeps[u] ? -1 : before;
      before += need[u] != kKept;
      if (slot[u] == s.slots - 1) s.running[seq[u]].y = before;
    }
    total += all;
  }
  __syncthreads();
  const int found = find_free<kReserveThreads>(p.refs, p.num_pages, used, total, s_waves[0], [&](int x, int page) { s.pages[x] = page; });
  __threadfence_block();
  __syncthreads();
  for (int base = 0; base < items; base += 4 * kReserveThreads) {
    int2 need[4], running[4];
    int page[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int item = min(base + u * kReserveThreads + tid, items - 1);
      need[u] = s.needs[item];
      running[u] = s.running[item / s.slots];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) page[u] = need[u].x != kKept && need[u].y < found ? s.pages[need[u].y] : 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int item = base + u * kReserveThreads + tid;
      if (item >= items) break;
      const int i = item / s.slots, x = item - i * s.slots;
      const bool there = wanted(p, i, &w) && (running[u].y <= found || running[u].x == running[u].y);
      if (there && need[u].x != kKept) {
        p.table[(size_t)i * p.max_pages + w.first + x] = page[u];
        p.refs[page[u]] = 1;
        if (need[u].x >= 0) atomicSub(p.refs + need[u].x, 1);
      }
      if (x == 0) {
        const bool moves = there && need[u].x >= 0 && w.begun;
        p.granted[i] = there ? w.count : 0;
        p.moves[2 * i] = moves ? need[u].x : -1;
        p.moves[2 * i + 1] = moves ? page[u] : -1;
      }
    }
  }
}

// The same where every thread has a sequence and that few pages: counts of a page's writers are kept in a hash table in LDS (open addressing, at most half full), needs in registers, so that
// three reads in a row are left: length, entries, counts.  What bounds it is those and the launch (512 sequences, five tokens each, pages of 16, 7.6 us; four 4.6; with each sequence a thread of
// the form above 14.6 and 6.9), and in pools that are nearly full the search (1.5 us for 16384 pages).
constexpr int kReserveSlots = 4, kHash = 2 * kReserveThreads;
__global__ __launch_bounds__(kReserveThreads)
void reserve_few_kernel(PageReserve p) {
  __shared__ int s_waves[2][kReserveThreads / 64], s_key[kHash], s_count[kHash], s_last[kHash], s_pages[kReserveThreads * kReserveSlots];
  const int tid = threadIdx.x;
  uint32_t used = in_use8(p.refs, 8 * tid, p.num_pages);
  Wanted w = {};
  const bool wants = tid < p.b && wanted(p, tid, &w);
  int entry[kReserveSlots], need[kReserveSlots];
#pragma unroll
  for (int x = 0; x < kReserveSlots; ++x) entry[x] = wants && w.first + x < w.last ? p.table[(size_t)tid * p.max_pages + w.first + x] : -1;
  int refs[kReserveSlots];
#pragma unroll
  for (int x = 0; x < kReserveSlots; ++x) refs[x] = is_page(entry[x], p.num_pages) ? p.refs[entry[x]] : 0;
  for (int x = tid; x < kHash; x += kReserveThreads) {
    s_key[x] = -1;
    s_count[x] = 0;
    s_last[x] = -1;
  }
  __syncthreads();
  const bool writes = wants && w.begun && refs[0] > 1;
  int at = 0;
  if (writes) {
    at = (int)((uint32_t)entry[0] * 2654435761u >> 21);
    for (;;) {
      const int key = atomicCAS(&s_key[at], -1, entry[0]);
      if (key == -1 || key == entry[0]) break;
      at = (at + 1) & (kHash - 1);
    }
    atomicAdd(&s_count[at], 1);
    atomicMax(&s_last[at], tid);
  }
  __syncthreads();
  const bool keeps = writes && s_count[at] == refs[0] && s_last[at] == tid;
  int needs = 0;
#pragma unroll
  for (int x = 0; x < kReserveSlots; ++x) {
    const bool there = is_page(entry[x], p.num_pages), begun = w.begun && x == 0;
    need[x] = !wants || w.first + x >= w.last || (begun && (!there || keeps)) || (there && refs[x] <= 1) ? kKept : there ? entry[x] : kMissing;
    needs += need[x] != kKept;
  }
  int total;
  const int running = before_me<kReserveThreads>(needs, s_waves[0], &total) + needs;
  const int found = find_free<kReserveThreads>(p.refs, p.num_pages, used, total, s_waves[1], [&](int x, int page) {
    if (x < total) s_pages[x] = page;
  });
  __syncthreads();
  if (tid >= p.b) return;
  int granted = 0, from = -1, to = -1;
  if (wants && (running <= found || (needs == 0 && !keeps))) {
    granted = w.count;
    int page_at = running - needs;
#pragma unroll
    for (int x = 0; x < kReserveSlots; ++x) {
      if (need[x] == kKept) continue;
      const int page = s_pages[page_at++];
      p.table[(size_t)tid * p.max_pages + w.first + x] = page;
      p.refs[page] = 1;
      if (need[x] >= 0) {
        atomicSub(p.refs + need[x], 1);
        if (w.begun && x == 0) { from = need[x]; to = page; }
      }
    }
  }
  p.granted[tid] = granted;
  p.moves[2 * tid] = from;
  p.moves[2 * tid + 1] = to;
}

// ---------------------------------------------------------------- compact
// With `used` pages in use, those from `used` on move, in order, to the free ones before it.
//
// Pools of up to kBitPages: a bit a page, in use or not, and the pages in use before every word of 32 are in LDS, of every workgroup: rank(page), the x-th free page and the x-th one in use (a binary
// search over the words, and in the word) say for each page, entry and move what it becomes without another workgroup's help.  The bits come from the counts, or, in pools so large that
// each workgroup would read many, from a launch before.  The launches and the reads in a row bound it (256 pages 5.9 us, 16384 8.3, 65536 11.3; by the three launches below 131072 12.6, so 16.7;
// 256 7.5).
constexpr int kBitPages = 1 << 16, kBitWords = kBitPages / 32, kReadPages = 1 << 14;
__device__ __forceinline__ uint32_t in_use32(const int32_t* refs, int word, int num_pages) {
  uint32_t bits = 0;
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (32 * word + 8 * x < num_pages) bits |= in_use8(refs, 32 * word + 8 * x, num_pages) << (8 * x);
  return bits;
}
__global__ __launch_bounds__(256)
void compact_bits_kernel(PageCompact p, uint32_t* bits) {      // a thread has four pages, eight neighbours a word
  const int first = 4 * (int)(blockIdx.x * 256u + threadIdx.x);
  uint32_t mine = 0;
  if (first + 4 <= p.num_pages) {
    const int4 a = *reinterpret_cast<const int4*>(p.refs_in + first);
    mine = (a.x > 0) | (a.y > 0) << 1 | (a.z > 0) << 2 | (a.w > 0) << 3;
  } else {
    for (int x = 0; first + x < p.num_pages; ++x) mine |= (uint32_t)(p.refs_in[first + x] > 0) << x;
  }
  mine <<= first & 31;
#pragma unroll
  for (int off = 1; off < 8; off <<= 1) mine |= __shfl_xor(mine, off);
  if ((threadIdx.x & 7) == 0 && first < p.num_pages) bits[first >> 5] = mine;
}
// The position of the x-th set bit (there are more than x).
__device__ __forceinline__ int nth_bit(uint32_t bits, int x) {
  int at = 0;
#pragma unroll
  for (int half = 16; half > 0; half >>= 1) {
    const int low = __popc(bits & ((1u << half) - 1));
    if (x >= low) {
      x -= low;
      at += half;
      bits >>= half;
    }
  }
  return at;
}
__global__ __launch_bounds__(256)
void compact_few_kernel(PageCompact p, const uint32_t* bits) {
  __shared__ uint32_t s_bits[kBitWords];
  __shared__ int s_rank[kBitWords], s_waves[2][4];
  const int tid = threadIdx.x, words = (p.num_pages + 31) / 32;
  for (int x = tid; x < words; x += 256) s_bits[x] = bits ? bits[x] : in_use32(p.refs_in, x, p.num_pages);
  __syncthreads();
  int used = 0;
  for (int base = 0, turn = 0; base < words; base += 1024, turn ^= 1) {
    int count[4], sum = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int word = base + 4 * tid + x;
      count[x] = word < words ? __popc(s_bits[word]) : 0;
      sum += count[x];
    }
    int all, before = used + before_me<256>(sum, s_waves[turn], &all);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (base + 4 * tid + x < words) s_rank[base + 4 * tid + x] = before;
      before += count[x];
    }
    used += all;
  }
  __syncthreads();
  auto rank = [&](int page) { return s_rank[page >> 5] + __popc(s_bits[page >> 5] & ((1u << (page & 31)) - 1)); };
  const int stay = used < p.num_pages ? rank(used) : used, moving = used - stay;
  // the last word before which there are no more than x pages in use (or free ones)
  auto tail = [&](int x) {               // the x-th page in use from `used` on
    x += stay;
    int word = 0;
    for (int half = kBitWords >> 1; half > 0; half >>= 1)
      if (word + half < words && s_rank[word + half] <= x) word += half;
    return 32 * word + nth_bit(s_bits[word], x - s_rank[word]);
  };
  auto hole = [&](int x) {
    int word = 0;
    for (int half = kBitWords >> 1; half > 0; half >>= 1)
      if (word + half < words && 32 * (word + half) - s_rank[word + half] <= x) word += half;
    return 32 * word + nth_bit(~s_bits[word], x - (32 * word - s_rank[word]));
  };
  const unsigned first = blockIdx.x * 256u + tid, step = gridDim.x * 256u;
  for (unsigned x = first; x < (unsigned)p.num_pages; x += step) {
    const int page = (int)x;
    int from = -1;
    if (page < used) from = s_bits[page >> 5] >> (page & 31) & 1 ? page : tail(page - rank(page));
    p.refs_out[page] = from < 0 ? 0 : p.refs_in[from];
  }
  for (unsigned x = first; x < (unsigned)p.moves_size; x += step)
    reinterpret_cast<int2*>(p.moves)[x] = (int)x < moving ? make_int2(tail((int)x), hole((int)x)) : make_int2(-1, -1);
  for (unsigned x = first; x < (unsigned)p.b * (unsigned)p.max_pages; x += step) {
    const int entry = p.table_in[x];
    int place = -1;
    if (is_page(entry, p.num_pages) && (s_bits[entry >> 5] >> (entry & 31) & 1)) place = entry < used ? entry : hole(rank(entry) - stay);
    p.table_out[x] = place;
  }
  if (first == 0) p.used[0] = used;
}

// Larger pools: three launches, pages in use of every chunk; every page's new place; tables and counts by it.
constexpr int kChunk = 2048;           // pages of a workgroup, eight a thread
struct CompactSpace { int32_t* counts; int32_t* place; size_t bytes; };
__host__ __device__ CompactSpace compact_space(int num_pages, void* at) {
  const size_t counts = (((size_t)(num_pages + kChunk - 1) / kChunk) * 4 + 15) & ~(size_t)15;
  return CompactSpace{static_cast<int32_t*>(at), reinterpret_cast<int32_t*>(static_cast<unsigned char*>(at) + counts),
                      counts + (((size_t)num_pages * 4 + 15) & ~(size_t)15)};
}

__global__ __launch_bounds__(256)
void compact_count_kernel(PageCompact p, void* workspace) {
  __shared__ int s_waves[4];
  int all;
  before_me<256>(__popc(in_use8(p.refs_in, blockIdx.x * kChunk + 8 * threadIdx.x, p.num_pages)), s_waves, &all);
  if (threadIdx.x == 0) compact_space(p.num_pages, workspace).counts[blockIdx.x] = all;
}

// place[page]: where it will be; -1: it is free; -2 - x: at the x-th hole, moves[x].
__global__ __launch_bounds__(256)
void compact_place_kernel(PageCompact p, void* workspace) {
  __shared__ int s_waves[4][4];
  const CompactSpace s = compact_space(p.num_pages, workspace);
  const int tid = threadIdx.x, chunks = gridDim.x;
  int before = 0, later = 0;
  for (int x = tid; x < chunks; x += 256) (x < (int)blockIdx.x ? before : later) += s.counts[x];
  int all_before, all_later;
  before_me<256>(before, s_waves[0], &all_before);
  before_me<256>(later, s_waves[1], &all_later);
  const int used = all_before + all_later;
  // pages in use before page `used`
  const int middle = used / kChunk;                      // its chunk
  int mine = 0;
  for (int x = tid; x < middle; x += 256) mine += s.counts[x];
  for (int x = middle * kChunk + tid; x < used; x += 256) mine += p.refs_in[x] > 0;
  int stay;
  before_me<256>(mine, s_waves[2], &stay);
  const int first = blockIdx.x * kChunk + 8 * tid;
  const uint32_t bits = in_use8(p.refs_in, first, p.num_pages);
  const int here = __popc(bits);
  int all;
  int rank = all_before + before_me<256>(here, s_waves[3], &all);      // pages in use before this one
  const int moving = used - stay;
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    const int page = first + x;
    if (page >= p.num_pages) break;
    const bool held = bits >> x & 1;
    int place = held ? page : -1;
    if (page < used && !held) p.moves[2 * (page - rank) + 1] = page;
    if (page >= used && held) {
      p.moves[2 * (rank - stay)] = page;
      place = -2 - (rank - stay);
    }
    s.place[page] = place;
    if (page >= moving && page < p.moves_size) p.moves[2 * page] = p.moves[2 * page + 1] = -1;
    rank += held;
  }
  if (blockIdx.x == 0 && tid == 0) p.used[0] = used;
}

__global__ __launch_bounds__(256)
void compact_apply_kernel(PageCompact p, void* workspace) {
  const CompactSpace s = compact_space(p.num_pages, workspace);
  const unsigned idx = blockIdx.x * 256u + threadIdx.x;
  const int used = p.used[0];
  if (idx < (unsigned)p.num_pages) {
    const int page = (int)idx, place = s.place[page];
    if (page >= used) p.refs_out[page] = 0;
    if (place >= 0) p.refs_out[place] = p.refs_in[page];
    if (place < -1) p.refs_out[p.moves[2 * (-2 - place) + 1]] = p.refs_in[page];
  }
  if (idx < (unsigned)p.b * (unsigned)p.max_pages) {
    const int entry = p.table_in[idx];
    int place = is_page(entry, p.num_pages) ? s.place[entry] : -1;
    if (place < -1) place = p.moves[2 * (-2 - place) + 1];
    p.table_out[idx] = place;
  }
}

// ---------------------------------------------------------------- copies of pages
// A workgroup a move at a time, 16 bytes (or 4, where a page's size asks for it) a thread.  HBM bounds it: 12320 moves of two pages of 4 KiB, 202 MB, 33.4 us = 6.05 TB/s (with stores that stay in L2
// 40.4; with loads that do not 36.4, and where eight moves copy the same page 11.1, so 7.2).
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
template <typename W>
__device__ __forceinline__ void copy_run(void* pool, uint32_t bytes, int from, int to) {
  const W* src = reinterpret_cast<const W*>(static_cast<const unsigned char*>(pool) + (size_t)from * bytes);
  W* dst = reinterpret_cast<W*>(static_cast<unsigned char*>(pool) + (size_t)to * bytes);
  const uint32_t words = bytes / sizeof(W);
  uint32_t x = threadIdx.x;
  for (; x + 768 < words; x += 1024) {
    const W a = src[x], b = src[x + 256], c = src[x + 512], d = src[x + 768];
    __builtin_nontemporal_store(a, dst + x);
    __builtin_nontemporal_store(b, dst + x + 256);
    __builtin_nontemporal_store(c, dst + x + 512);
    __builtin_nontemporal_store(d, dst + x + 768);
  }
  for (; x < words; x += 256) __builtin_nontemporal_store(src[x], dst + x);
}
constexpr int kCopyGrid = 16384;
__global__ __launch_bounds__(256)
void copy_pages_kernel(PageCopy p) {
  for (int m = blockIdx.x; m < p.m; m += gridDim.x) {
    const int from = p.moves[2 * m], to = p.moves[2 * m + 1];
    if (!is_page(from, p.num_pages) || !is_page(to, p.num_pages) || from == to) continue;
    for (int x = 0; x < p.pools; ++x)
      if (p.page_bytes[x] % 16 == 0) copy_run<u32x4>(p.pool[x], p.page_bytes[x], from, to);
      else copy_run<uint32_t>(p.pool[x], p.page_bytes[x], from, to);
  }
}

}  // namespace

hipError_t launch_fork(const PageFork& p, hipStream_t st) {
  hipLaunchKernelGGL(fork_kernel, dim3(((unsigned)((p.b_out + kRun - 1) / kRun) * (unsigned)p.max_pages + 255) / 256), dim3(256), 0, st, p);
  return hipGetLastError();
}

hipError_t launch_free(const PageFree& p, hipStream_t st) {
  hipLaunchKernelGGL(free_kernel, dim3(((unsigned)((p.b + kRun - 1) / kRun) * (unsigned)p.max_pages + 255) / 256), dim3(256), 0, st, p);
  return hipGetLastError();
}

size_t reserve_workspace_bytes(int b, int n, int num_pages, int page_size) { return reserve_space(b, n, num_pages, page_size, nullptr).bytes; }

hipError_t launch_reserve(const PageReserve& p, void* workspace, hipStream_t st) {
  if (p.b <= kReserveThreads && reserve_space(p.b, p.n, p.num_pages, p.page_size, nullptr).slots <= kReserveSlots)
    hipLaunchKernelGGL(reserve_few_kernel, dim3(1), dim3(kReserveThreads), 0, st, p);
  else
    hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kReserveThreads), 0, st, p, workspace);
  return hipGetLastError();
}

size_t compact_workspace_bytes(int num_pages) { return compact_space(num_pages, nullptr).bytes; }

hipError_t launch_compact(const PageCompact& p, void* workspace, hipStream_t st) {
  const unsigned entries = (unsigned)p.b * (unsigned)p.max_pages, items = entries > (unsigned)p.num_pages ? entries : (unsigned)p.num_pages;
  if (p.num_pages <= kBitPages) {
    uint32_t* bits = nullptr;
    if (p.num_pages > kReadPages) {
      bits = static_cast<uint32_t*>(workspace);
      hipLaunchKernelGGL(compact_bits_kernel, dim3(((unsigned)p.num_pages + 1023) / 1024), dim3(256), 0, st, p, bits);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    const unsigned groups = (items + 255) / 256;
    hipLaunchKernelGGL(compact_few_kernel, dim3(groups < 256 ? groups : 256), dim3(256), 0, st, p, bits);
    return hipGetLastError();
  }
  const unsigned chunks = ((unsigned)p.num_pages + kChunk - 1) / kChunk;
  hipLaunchKernelGGL(compact_count_kernel, dim3(chunks), dim3(256), 0, st, p, workspace);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_place_kernel, dim3(chunks), dim3(256), 0, st, p, workspace);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_apply_kernel, dim3((items + 255) / 256), dim3(256), 0, st, p, workspace);
  return hipGetLastError();
}

hipError_t launch_copy_pages(const PageCopy& p, hipStream_t st) {
  hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)(p.m < kCopyGrid ? p.m : kCopyGrid)), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace mqa
