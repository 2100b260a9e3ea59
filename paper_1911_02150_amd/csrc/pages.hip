// Who holds which page of a pool.  refs[page]: how many entries of tables name it; a page with none (or fewer) is free.  Pages are given out from the lowest
// free one on, so that what a call does depends on its arguments alone.
#include "paged.hpp"

namespace mqa {
namespace {

__device__ __forceinline__ bool is_page(int entry, int num_pages) { return (unsigned)entry < (unsigned)num_pages; }
__device__ __forceinline__ int pages_of(int len, int page_size) { return (int)(((unsigned)len + (unsigned)page_size - 1) / (unsigned)page_size); }

// ---------------------------------------------------------------- fork, free: a thread an entry
__global__ __launch_bounds__(256)
void fork_kernel(PageFork p) {
  const unsigned idx = blockIdx.x * 256u + threadIdx.x;
  if (idx >= (unsigned)p.b_out * (unsigned)p.max_pages) return;
  const int j = (int)(idx / (unsigned)p.max_pages), x = (int)(idx - (unsigned)j * (unsigned)p.max_pages);
  const int parent = p.parents[j];
  int len = 0, entry = -1;
  if ((unsigned)parent < (unsigned)p.b_in) {
    len = min(max(p.lens_in[parent], 0), p.max_pages * p.page_size);
    if (x < pages_of(len, p.page_size)) entry = p.table_in[(size_t)parent * p.max_pages + x];
    if (!is_page(entry, p.num_pages)) entry = -1;
  }
  if (entry >= 0) atomicAdd(p.refs + entry, 1);
  p.table_out[idx] = entry;
  if (x == 0) p.lens_out[j] = len;
}

__global__ __launch_bounds__(256)
void free_kernel(PageFree p) {
  const unsigned idx = blockIdx.x * 256u + threadIdx.x;
  if (idx >= (unsigned)p.b * (unsigned)p.max_pages) return;
  const int i = (int)(idx / (unsigned)p.max_pages), x = (int)(idx - (unsigned)i * (unsigned)p.max_pages);
  const int len = min(max(p.lens[i], 0), p.max_pages * p.page_size);
  if (x < pages_of(len, p.page_size)) return;
  const int entry = p.table[idx];
  if (is_page(entry, p.num_pages)) atomicSub(p.refs + entry, 1);
  if (entry != -1) p.table[idx] = -1;
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

// ---------------------------------------------------------------- reserve
// One workgroup, in steps:
//  1. of every page that sequences are about to write behind rows that others share: how many are, and the last of them
//  2. what every sequence needs: per page of its new positions nothing (kKept), a page (kMissing), or a page in place of a shared one (that one's number);
//     and how many pages that makes, running over the sequences
//  3. as many free pages as are needed, or as there are
//  4. to the sequences whose running number is there: their pages
// (Step 4 reads what step 2 has written down and no counts, since it changes them.)
constexpr int kReserveThreads = 1024;
constexpr int kKept = -2, kMissing = -1;

struct ReserveSpace {
  int2* writers;       // [num_pages]: how many, the last (written before they are read, where they are read)
  int32_t* needs;      // [b, slots]
  int32_t* running;    // [b]
  int32_t* pages;      // free ones
  int slots;
  size_t bytes;
};
__host__ __device__ ReserveSpace reserve_space(int b, int n, int num_pages, int page_size, void* at) {
  ReserveSpace s;
  s.slots = (int)((n + (long long)page_size - 2) / page_size) + 1;      // pages that n rows reach, at most
  const size_t writers = ((size_t)num_pages * 8 + 15) & ~(size_t)15, needs = ((size_t)b * s.slots * 4 + 15) & ~(size_t)15, running = ((size_t)b * 4 + 15) & ~(size_t)15;
  unsigned char* const p = static_cast<unsigned char*>(at);
  s.writers = reinterpret_cast<int2*>(p);
  s.needs = reinterpret_cast<int32_t*>(p + writers);
  s.running = reinterpret_cast<int32_t*>(p + writers + needs);
  s.pages = reinterpret_cast<int32_t*>(p + writers + needs + running);
  s.bytes = writers + needs + running + (((size_t)num_pages * 4 + 15) & ~(size_t)15);
  return s;
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
  for (int i = tid; i < p.b; i += kReserveThreads) {
    const int page = begun_page(i);
    if (page >= 0) s.writers[page] = make_int2(0, -1);
  }
  __threadfence_block();
  __syncthreads();
  for (int i = tid; i < p.b; i += kReserveThreads) {
    const int page = begun_page(i);
    if (page >= 0) {
      atomicAdd(&s.writers[page].x, 1);
      atomicMax(&s.writers[page].y, i);
    }
  }
  __threadfence_block();
  __syncthreads();
  int total = 0;
  for (int base = 0, turn = 0; base < p.b; base += kReserveThreads, turn ^= 1) {
    const int i = base + tid;
    int needs = 0;
    bool keeps = false;
    if (i < p.b && wanted(p, i, &w)) {
      for (int x = w.first; x < w.last; ++x) {
        const int entry = p.table[(size_t)i * p.max_pages + x];
        const bool there = is_page(entry, p.num_pages);
        const int refs = there ? p.refs[entry] : 0;
        int need = there && refs <= 1 ? kKept : there ? entry : kMissing;
        if (w.begun && x == w.first) {
          if (!there) need = kKept;                    // (rows on no page: they stay nowhere)
          if (need >= 0) {
            // (past L1, which the atomics do not go through)
            const int others = __hip_atomic_load(&s.writers[entry].x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (others == refs && __hip_atomic_load(&s.writers[entry].y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i) { need = kKept; keeps = true; }
          }
        }
        s.needs[(size_t)i * s.slots + (x - w.first)] = need;
        needs += need != kKept;
      }
    }
    int all;
    const int before = before_me<kReserveThreads>(needs, s_waves[turn], &all);
    // (who keeps a page that others are about to leave may do so only if they do)
    if (i < p.b) s.running[i] = needs == 0 && !keeps ? 0 : total + before + needs;
    total += all;
  }
  int found = 0;
  for (int base = 0, turn = 0; base < p.num_pages && found < total; base += kReserveThreads, turn ^= 1) {
    __syncthreads();
    const int page = base + tid;
    const bool free = page < p.num_pages && p.refs[page] <= 0;
    int all;
    const int at = found + before_me<kReserveThreads>(free, s_waves[turn], &all);
    if (free) s.pages[at] = page;
    found += all;
  }
  __threadfence_block();
  __syncthreads();
  for (int i = tid; i < p.b; i += kReserveThreads) {
    int granted = 0, from = -1, to = -1;
    if (wanted(p, i, &w) && s.running[i] <= found) {
      granted = w.count;
      int at = s.running[i];
      for (int x = w.last - 1; x >= w.first; --x) {      // (from its last page backwards)
        const int need = s.needs[(size_t)i * s.slots + (x - w.first)];
        if (need == kKept) continue;
        const int page = s.pages[--at];
        p.table[(size_t)i * p.max_pages + x] = page;
        p.refs[page] = 1;
        if (need >= 0) {
          atomicSub(p.refs + need, 1);
          if (w.begun && x == w.first) { from = need; to = page; }
        }
      }
    }
    p.granted[i] = granted;
    p.moves[2 * i] = from;
    p.moves[2 * i + 1] = to;
  }
}

// ---------------------------------------------------------------- compact
// With `used` pages in use, those from `used` on move, in order, to the free ones before it.  Three launches: pages in use of every chunk; every page's new place; tables
// and counts by it.
constexpr int kChunk = 2048;           // pages of a workgroup, eight a thread
struct CompactSpace { int32_t* counts; int32_t* place; size_t bytes; };
__host__ __device__ CompactSpace compact_space(int num_pages, void* at) {
  const size_t counts = (((size_t)(num_pages + kChunk - 1) / kChunk) * 4 + 15) & ~(size_t)15;
  return CompactSpace{static_cast<int32_t*>(at), reinterpret_cast<int32_t*>(static_cast<unsigned char*>(at) + counts),
                      counts + (((size_t)num_pages * 4 + 15) & ~(size_t)15)};
}

__device__ __forceinline__ int in_use(const PageCompact& p, int first, uint32_t* bits) {      // of eight pages
  int sum = 0;
  *bits = 0;
#pragma unroll
  for (int x = 0; x < 8; ++x)
    if (first + x < p.num_pages && p.refs_in[first + x] > 0) {
      ++sum;
      *bits |= 1u << x;
    }
  return sum;
}

__global__ __launch_bounds__(256)
void compact_count_kernel(PageCompact p, void* workspace) {
  __shared__ int s_waves[4];
  uint32_t bits;
  int all;
  before_me<256>(in_use(p, blockIdx.x * kChunk + 8 * threadIdx.x, &bits), s_waves, &all);
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
  uint32_t bits;
  const int here = in_use(p, first, &bits);
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
// A workgroup a move at a time, 16 bytes (or 4, where a page's size asks for it) a thread.
template <typename W>
__device__ __forceinline__ void copy_run(void* pool, uint32_t bytes, int from, int to) {
  const W* src = reinterpret_cast<const W*>(static_cast<const unsigned char*>(pool) + (size_t)from * bytes);
  W* dst = reinterpret_cast<W*>(static_cast<unsigned char*>(pool) + (size_t)to * bytes);
  for (uint32_t x = threadIdx.x; x < bytes / sizeof(W); x += 256) dst[x] = src[x];
}
__global__ __launch_bounds__(256)
void copy_pages_kernel(PageCopy p) {
  for (int m = blockIdx.x; m < p.m; m += gridDim.x) {
    const int from = p.moves[2 * m], to = p.moves[2 * m + 1];
    if (!is_page(from, p.num_pages) || !is_page(to, p.num_pages) || from == to) continue;
    for (int x = 0; x < p.pools; ++x)
      if (p.page_bytes[x] % 16 == 0) copy_run<uint4>(p.pool[x], p.page_bytes[x], from, to);
      else copy_run<uint32_t>(p.pool[x], p.page_bytes[x], from, to);
  }
}

}  // namespace

hipError_t launch_fork(const PageFork& p, hipStream_t st) {
  hipLaunchKernelGGL(fork_kernel, dim3(((unsigned)p.b_out * (unsigned)p.max_pages + 255) / 256), dim3(256), 0, st, p);
  return hipGetLastError();
}

hipError_t launch_free(const PageFree& p, hipStream_t st) {
  hipLaunchKernelGGL(free_kernel, dim3(((unsigned)p.b * (unsigned)p.max_pages + 255) / 256), dim3(256), 0, st, p);
  return hipGetLastError();
}

size_t reserve_workspace_bytes(int b, int n, int num_pages, int page_size) { return reserve_space(b, n, num_pages, page_size, nullptr).bytes; }

hipError_t launch_reserve(const PageReserve& p, void* workspace, hipStream_t st) {
  hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kReserveThreads), 0, st, p, workspace);
  return hipGetLastError();
}

size_t compact_workspace_bytes(int num_pages) { return compact_space(num_pages, nullptr).bytes; }

hipError_t launch_compact(const PageCompact& p, void* workspace, hipStream_t st) {
  const unsigned chunks = ((unsigned)p.num_pages + kChunk - 1) / kChunk;
  hipLaunchKernelGGL(compact_count_kernel, dim3(chunks), dim3(256), 0, st, p, workspace);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_place_kernel, dim3(chunks), dim3(256), 0, st, p, workspace);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const unsigned entries = (unsigned)p.b * (unsigned)p.max_pages, items = entries > (unsigned)p.num_pages ? entries : (unsigned)p.num_pages;
  hipLaunchKernelGGL(compact_apply_kernel, dim3((items + 255) / 256), dim3(256), 0, st, p, workspace);
  return hipGetLastError();
}

hipError_t launch_copy_pages(const PageCopy& p, hipStream_t st) {
  hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)(p.m < 16384 ? p.m : 16384)), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace mqa
