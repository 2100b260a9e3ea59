// Attention of the newest tokens of every sequence over a paged cache.
//
// Per (sequence, K/V head) the R = n * h / h_kv query rows share the K and V rows; row r is query j = r / (h / h_kv), which sees the positions below
// lens - (n - 1 - j):
//   logits[r,p] = scale * sum_c q[r,c] K[p,c];  weights = softmax over p;  o[r,:] = sum_p weights[r,p] V[p,:]
// Positions on pages that hold nothing have weight 0, and a row that sees nothing is 0.
#include "paged.hpp"

namespace mqa {
namespace {

constexpr int kThreads = 256;
constexpr int kScalarRows = 8;            // query rows of a pass of the scalar form

// A run of tiles of one unit.
struct Segment {
  int i, e, row0;          // sequence, head, first query row of the block
  int L;                   // the sequence's length
  int begin, end;          // positions
  int slot;                // where its partial states go; -1: the segment is the whole unit
};

__device__ __forceinline__ size_t row_offset(const PagedDecode& p, int i, int e, int r) {      // of q and o, in rows
  const int group = p.h / p.c.h_kv;
  return ((size_t)i * p.n + r / group) * p.h + (size_t)e * group + r % group;
}
__device__ __forceinline__ int row_limit(const PagedDecode& p, int L, int r) {                 // the first position that row r does not see
  return max(0, L - (p.n - 1 - r / (p.h / p.c.h_kv)));
}
__device__ __forceinline__ size_t logits_pitch(const PagedDecode& p) { return (size_t)((p.c.positions() + kPagedTile - 1) / kPagedTile) * kPagedTile; }

// The plain form of a segment, rows r0 .. r0 + nr - 1 of the group (nr <= 8): float32 products, any widths.  What is not seen is never multiplied, so that
// it may hold infinities and NaN.  LDS in floats: q, one tile of K or V rows (at the end the parts of the outputs), weights, states.
__host__ __device__ constexpr size_t scalar_lds_floats(int k, int v) {
  const int w = (k > v ? k : v) + 4;
  const size_t tile = (size_t)kPagedTile * w, parts = 8192;
  return (size_t)kScalarRows * k + (tile > parts ? tile : parts) + kScalarRows * kPagedTile + 3 * kScalarRows + kPagedTile + kScalarRows;
}

__device__ __forceinline__ float4 cache4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 cache4(const uint16_t* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
}

template <typename T>
__device__ void scalar_segment(const PagedDecode& p, const Segment& s, int r0, int nr, float* smem) {
  const int tid = threadIdx.x;
  const int k = p.c.k, v = p.c.v, k4 = k >> 2, v4 = v >> 2, pitch = (k > v ? k : v) + 4;
  float* sq = smem;                                                  // [8][k]
  float* st = sq + kScalarRows * k;                                  // [32][pitch]
  const size_t tile = (size_t)kPagedTile * pitch;
  float* sw = st + (tile > 8192 ? tile : 8192);                      // [8][32] logits, then weights
  float* s_m = sw + kScalarRows * kPagedTile;
  float* s_l = s_m + kScalarRows;
  float* s_a = s_l + kScalarRows;
  int* s_row = reinterpret_cast<int*>(s_a + kScalarRows);            // [32] rows of the pool
  int* s_lim = s_row + kPagedTile;                                   // [8]
  const int32_t* table = p.c.table + (size_t)s.i * p.c.max_pages;
  const T* K = static_cast<const T*>(p.c.K);
  const T* V = static_cast<const T*>(p.c.V);
  __syncthreads();
  for (int idx = tid; idx < nr * k4; idx += kThreads) {
    const int r = idx / k4;
    float4 x = reinterpret_cast<const float4*>(p.q + row_offset(p, s.i, s.e, r0 + r) * k)[idx - r * k4];
    x.x *= p.qscale; x.y *= p.qscale; x.z *= p.qscale; x.w *= p.qscale;
    reinterpret_cast<float4*>(sq)[idx] = x;
  }
  if (tid < kScalarRows) {
    s_m[tid] = -INFINITY;
    s_l[tid] = 0.f;
    s_lim[tid] = tid < nr ? row_limit(p, s.L, r0 + tid) : 0;
  }
  float4 acc[kScalarRows];
#pragma unroll
  for (int j = 0; j < kScalarRows; ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
  const int PG = kThreads / v4, c4 = tid % v4, pg = tid / v4;        // weighted sum: a thread has four columns and every PG-th position
  const int dpos = tid & 31, drow = tid >> 5;                        // logits: a thread has a position and a row
  for (int p0 = s.begin; p0 < s.end; p0 += kPagedTile) {
    __syncthreads();
    if (tid < kPagedTile) s_row[tid] = p0 + tid < s.end ? paged_row(p.c, table, s.e, p0 + tid) : -1;
    __syncthreads();
    for (int idx = tid; idx < kPagedTile * k4; idx += kThreads) {
      const int r = idx / k4, c = idx - r * k4;
      const int row = s_row[r];
      *reinterpret_cast<float4*>(st + r * pitch + 4 * c) = row < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : cache4(K + (size_t)row * k + 4 * c);
    }
    __syncthreads();
    if (drow < nr) {
      float dot = -INFINITY;
      if (s_row[dpos] >= 0 && p0 + dpos < s_lim[drow]) {
        const float4 *kr = reinterpret_cast<const float4*>(st + dpos * pitch), *qr = reinterpret_cast<const float4*>(sq + drow * k);
        dot = 0.f;
        for (int c = 0; c < k4; ++c) {
          const float4 x = kr[c], y = qr[c];
          dot = fmaf(y.x, x.x, fmaf(y.y, x.y, fmaf(y.z, x.z, fmaf(y.w, x.w, dot))));
        }
      }
      sw[drow * kPagedTile + dpos] = dot;
      if (p.logits && p0 + dpos < s.end)
        p.logits[(((size_t)s.i * p.c.h_kv + s.e) * p.R + r0 + drow) * logits_pitch(p) + p0 + dpos] = dot;
    }
    __syncthreads();
    for (int idx = tid; idx < kPagedTile * v4; idx += kThreads) {
      const int r = idx / v4, c = idx - r * v4;
      const int row = s_row[r];
      *reinterpret_cast<float4*>(st + r * pitch + 4 * c) = row < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : cache4(V + (size_t)row * v + 4 * c);
    }
    if (drow < nr) {                                                 // (the 32 threads of a row are half a wave)
      const float z = sw[drow * kPagedTile + dpos];
      float zmax = z;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) zmax = fmaxf(zmax, __shfl_xor(zmax, off));
      const float mold = s_m[drow], mnew = fmaxf(mold, zmax), mref = mnew == -INFINITY ? 0.f : mnew;
      const float w = z == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(z - mref);
      float sum = w;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
      sw[drow * kPagedTile + dpos] = w;
      if (dpos == 0) {
        const float alpha = __builtin_amdgcn_exp2f(mold - mref);
        s_a[drow] = alpha;
        s_l[drow] = s_l[drow] * alpha + sum;
        s_m[drow] = mnew;
      }
    }
    __syncthreads();
    if (pg < PG) {
#pragma unroll
      for (int j = 0; j < kScalarRows; ++j) {
        const float a = j < nr ? s_a[j] : 0.f;
        acc[j].x *= a; acc[j].y *= a; acc[j].z *= a; acc[j].w *= a;
      }
      for (int r = pg; r < kPagedTile; r += PG) {
        if (s_row[r] < 0) continue;
        const float4 x = reinterpret_cast<const float4*>(st + r * pitch)[c4];
#pragma unroll
        for (int j = 0; j < kScalarRows; ++j)
          if (j < nr && p0 + r < s_lim[j]) {
            const float w = sw[j * kPagedTile + r];
            acc[j].x = fmaf(w, x.x, acc[j].x); acc[j].y = fmaf(w, x.y, acc[j].y); acc[j].z = fmaf(w, x.z, acc[j].z); acc[j].w = fmaf(w, x.w, acc[j].w);
          }
      }
    }
  }
  __syncthreads();
  // the positions' groups, up to 32 KiB of them at a time: 8192 floats hold 8192 / (8 v) groups
  const int held = min(PG, 8192 / (kScalarRows * v));
  float4 sums[kScalarRows];
#pragma unroll
  for (int j = 0; j < kScalarRows; ++j) sums[j] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int g0 = 0; g0 < PG; g0 += held) {
    if (pg >= g0 && pg < min(PG, g0 + held))
#pragma unroll
      for (int j = 0; j < kScalarRows; ++j) reinterpret_cast<float4*>(st + ((size_t)(pg - g0) * kScalarRows + j) * v)[c4] = acc[j];
    __syncthreads();
    if (tid < v4)
      for (int g = 0; g < min(held, PG - g0); ++g)
#pragma unroll
        for (int j = 0; j < kScalarRows; ++j) {
          const float4 x = reinterpret_cast<const float4*>(st + ((size_t)g * kScalarRows + j) * v)[tid];
          sums[j].x += x.x; sums[j].y += x.y; sums[j].z += x.z; sums[j].w += x.w;
        }
    __syncthreads();
  }
  if (tid < v4)
#pragma unroll
    for (int j = 0; j < kScalarRows; ++j) {
      if (j >= nr) break;
      float4 a = sums[j];
      if (s.slot < 0) {
        const float inv = s_m[j] == -INFINITY && s_l[j] == 0.f ? 0.f : 1.f / s_l[j];
        a.x *= inv; a.y *= inv; a.z *= inv; a.w *= inv;
        reinterpret_cast<float4*>(p.o + row_offset(p, s.i, s.e, r0 + j) * v)[tid] = a;
      } else {
        reinterpret_cast<float4*>(p.part_o + ((size_t)s.slot * p.block_rows + r0 + j - s.row0) * v)[tid] = a;
      }
    }
  if (tid < nr) {
    if (s.slot >= 0) {
      p.part_m[(size_t)s.slot * p.block_rows + r0 + tid - s.row0] = s_m[tid];
      p.part_l[(size_t)s.slot * p.block_rows + r0 + tid - s.row0] = s_l[tid];
    } else if (p.stats) {
      float* stat = p.stats + (((size_t)s.i * p.c.h_kv + s.e) * p.R + r0 + tid) * 2;
      stat[0] = s_m[tid] == -INFINITY ? 0.f : s_m[tid];
      stat[1] = s_m[tid] == -INFINITY && s_l[tid] == 0.f ? 0.f : 1.f / s_l[tid];
    }
  }
}

// ---------------------------------------------------------------- the list of work
__device__ __forceinline__ int tiles_of(const PagedDecode& p, int i) { return (paged_length(p.c, p.lens[i]) + kPagedTile - 1) / kPagedTile; }

// The workgroups that share `total` tiles: as many as have kLeastTiles each, one at least.
constexpr int kLeastTiles = 4;
__device__ __forceinline__ long long sharing(const PagedDecode& p, long long total) { return max(1ll, min((long long)p.W, total / kLeastTiles)); }
// Workgroup w of W has the tiles w * total / W up to the next one's; this is the one that has tile g.
__device__ __forceinline__ int workgroup_of(long long g, long long total, long long W) { return (int)(((g + 1) * W - 1) / total); }

// Tiles of the sequences before each one, all threads of the workgroup together: thread t has sequences t * per up to the next one's.
__device__ __forceinline__ int tiles_before_me(const PagedDecode& p, int per, int* s_waves, int* total, int* mine) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int sum = 0;
  for (int x = 0; x < per; ++x) {
    const long long i = (long long)tid * per + x;
    if (i < p.b) sum += tiles_of(p, (int)i);
  }
  int incl = sum;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(incl, off);
    if (lane >= off) incl += y;
  }
  if (lane == 63) s_waves[wave] = incl;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before += s_waves[w];
    all += s_waves[w];
  }
  *total = all;
  *mine = sum;
  return before + incl - sum;
}

// Runs `work` over the segments of this workgroup.
template <typename Work>
__device__ __forceinline__ void for_segments(const PagedDecode& p, Work&& work) {
  __shared__ int s_waves[kThreads / 64];
  __shared__ int s_at[2];
  const int tid = threadIdx.x;
  const long long units = (long long)p.c.h_kv * p.blocks;       // of a sequence
  if (!p.split) {                                               // a unit each
    const long long u = blockIdx.x;
    Segment s;
    s.i = (int)(u / units);
    s.e = (int)(u % units) / p.blocks;
    s.row0 = (int)(u % p.blocks) * p.block_rows;
    s.L = paged_length(p.c, p.lens[s.i]);
    s.begin = 0;
    s.end = s.L;
    s.slot = -1;
    work(s);
    return;
  }
  const int per = (p.b + kThreads - 1) / kThreads;
  int tiles, mine;
  const int before = tiles_before_me(p, per, s_waves, &tiles, &mine);
  if (blockIdx.x == 0) {                                        // for the merge
    int at = before;
    for (int x = 0; x < per; ++x) {
      const long long i = (long long)tid * per + x;
      if (i > p.b) break;
      p.starts[i] = at;
      if (i < p.b) at += tiles_of(p, (int)i);
    }
    if (tid == 0) p.starts[p.b] = tiles;
  }
  const long long total = tiles * units, W = sharing(p, total), w = blockIdx.x;
  if (w >= W || total == 0) return;
  long long at = w * total / W;
  const long long end = (w + 1) * total / W;
  if (before * units <= at && at < (before + mine) * units) {   // one thread: its sequences hold the first tile
    int b0 = before;
    for (int x = 0; x < per; ++x) {
      const int i = tid * per + x, t = tiles_of(p, i);
      if (at < (b0 + t) * units) {
        s_at[0] = i;
        s_at[1] = b0;
        break;
      }
      b0 += t;
    }
  }
  __syncthreads();
  int i = s_at[0], first = s_at[1];
  while (at < end) {
    const int L = paged_length(p.c, p.lens[i]), t = (L + kPagedTile - 1) / kPagedTile;
    const long long off = at - first * units;
    if (off >= t * units) {                                     // the next sequence
      first += t;
      ++i;
      continue;
    }
    const int u = (int)(off / t), tile0 = (int)(off - (long long)u * t), count = (int)min((long long)(t - tile0), end - at);
    Segment s;
    s.i = i;
    s.e = u / p.blocks;
    s.row0 = (u % p.blocks) * p.block_rows;
    s.L = L;
    s.begin = tile0 * kPagedTile;
    s.end = min(L, (tile0 + count) * kPagedTile);
    s.slot = count == t ? -1 : 2 * (int)w + (tile0 > 0 ? 0 : 1);
    work(s);
    at += count;
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads)
void paged_scalar_kernel(PagedDecode p) {
  extern __shared__ __align__(16) float smem[];
  for_segments(p, [&](const Segment& s) { scalar_segment<T>(p, s, s.row0, min(p.R - s.row0, kScalarRows), smem); });
}

// ---------------------------------------------------------------- merge
// The slots of a unit that several workgroups had: the first one's second, then the others' first.
struct Slots { int w0, w1; };
__device__ __forceinline__ Slots slots_of(const PagedDecode& p, int i, int e, int block, bool* empty) {
  const int t0 = p.starts[i], t = p.starts[i + 1] - t0;
  const long long units = (long long)p.c.h_kv * p.blocks, total = p.starts[p.b] * units;
  *empty = t == 0;
  if (t == 0) return Slots{0, 0};
  const long long W = sharing(p, total), g = t0 * units + ((long long)e * p.blocks + block) * t;
  return Slots{workgroup_of(g, total, W), workgroup_of(g + t - 1, total, W)};
}
__device__ __forceinline__ size_t slot_of(const Slots& s, int x) { return (size_t)(x == 0 ? 2 * s.w0 + 1 : 2 * (s.w0 + x)); }

// With (m_s, l_s, acc_s) the partial states: M = max m_s, l = sum l_s 2^(m_s - M), o = sum acc_s 2^(m_s - M) / l.  A workgroup has `rows` rows of a unit,
// thread = (four columns, row, slot group).
__global__ __launch_bounds__(256)
void paged_merge_kernel(PagedDecode p, int rows) {
  __shared__ float s_m[256], s_l[256];
  __shared__ float4 s_a[256];
  const int v4 = p.c.v >> 2, tid = threadIdx.x;
  const int pieces = (p.block_rows + rows - 1) / rows;
  const long long u = (long long)blockIdx.x / pieces;
  const int block = (int)(u % p.blocks), e = (int)(u / p.blocks % p.c.h_kv), i = (int)(u / p.blocks / p.c.h_kv);
  const int groups = 256 / (v4 * rows);
  const int c4 = tid % v4, row = tid / v4 % rows, sg = tid / v4 / rows;
  const int rb = (int)(blockIdx.x % pieces) * rows + row, r = block * p.block_rows + rb;      // in the block, and in the group
  bool empty;
  const Slots s = slots_of(p, i, e, block, &empty);
  if (!empty && s.w0 == s.w1) return;                    // finished by its workgroup
  const bool mine = sg < groups && rb < p.block_rows && r < p.R;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  float M = -INFINITY, l = 0.f;
  const int count = empty ? 0 : s.w1 - s.w0 + 1;
  if (mine)
    for (int x0 = sg; x0 < count; x0 += 4 * groups) {
      float pm[4], pl[4];
      float4 po[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const size_t at = slot_of(s, min(x0 + x * groups, count - 1)) * p.block_rows + rb;
        pm[x] = p.part_m[at];
        pl[x] = p.part_l[at];
        po[x] = reinterpret_cast<const float4*>(p.part_o + at * p.c.v)[c4];
      }
      float Mn = M;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (x0 + x * groups < count) Mn = fmaxf(Mn, pm[x]);
      const float ref = Mn == -INFINITY ? 0.f : Mn, f0 = __builtin_amdgcn_exp2f(M - ref);
      a.x *= f0; a.y *= f0; a.z *= f0; a.w *= f0;
      l *= f0;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (x0 + x * groups < count) {
          const float f = __builtin_amdgcn_exp2f(pm[x] - ref);
          a.x += f * po[x].x; a.y += f * po[x].y; a.z += f * po[x].z; a.w += f * po[x].w;
          l += f * pl[x];
        }
      M = Mn;
    }
  if (groups > 1) {
    s_m[tid] = M;
    s_l[tid] = l;
    s_a[tid] = a;
    __syncthreads();
    if (sg != 0) return;
    const int per = v4 * rows;
    for (int g = 1; g < groups; ++g) M = fmaxf(M, s_m[g * per + tid]);
    const float ref = M == -INFINITY ? 0.f : M;
    a = make_float4(0.f, 0.f, 0.f, 0.f);
    l = 0.f;
    for (int g = 0; g < groups; ++g) {
      const float f = __builtin_amdgcn_exp2f(s_m[g * per + tid] - ref);
      const float4 x = s_a[g * per + tid];
      a.x += f * x.x; a.y += f * x.y; a.z += f * x.z; a.w += f * x.w;
      l += f * s_l[g * per + tid];
    }
  }
  if (!mine || sg != 0) return;
  const float inv = M == -INFINITY && l == 0.f ? 0.f : 1.f / l;
  a.x *= inv; a.y *= inv; a.z *= inv; a.w *= inv;
  reinterpret_cast<float4*>(p.o + row_offset(p, i, e, r) * p.c.v)[c4] = a;
  if (p.stats && c4 == 0) {
    float* stat = p.stats + (((size_t)i * p.c.h_kv + e) * p.R + r) * 2;
    stat[0] = M == -INFINITY ? 0.f : M;
    stat[1] = inv;
  }
}

// scores_out[p] = (p is older than this step's tokens ? scores_in[p] : 0) + sum over the rows of their weights at p.  A thread has a position.
__global__ __launch_bounds__(256)
void paged_scores_kernel(PagedDecode p, int chunks) {
  const int g = blockIdx.x / chunks, pos = (int)(blockIdx.x % chunks) * 256 + threadIdx.x, i = g / p.c.h_kv;
  const int L = paged_length(p.c, p.lens[i]);
  if (pos >= L) return;
  const size_t pitch = logits_pitch(p), at = (size_t)g * p.c.positions() + pos;
  const float* z = p.logits + (size_t)g * p.R * pitch + pos;
  const float* stat = p.stats + (size_t)g * p.R * 2;
  float sum = 0.f;
  for (int r = 0; r < p.R; ++r) sum += __builtin_amdgcn_exp2f(z[r * pitch] - stat[2 * r]) * stat[2 * r + 1];
  p.scores_out[at] = (p.scores_in && pos < L - p.n ? p.scores_in[at] : 0.f) + sum;
}

}  // namespace

constexpr int kPagedWorkgroups = 512;

// The parts of a call's workspace, each on 16 bytes; their size in all.
static size_t lay_out(PagedDecode* p, const PagedPlan& pl, float* at) {
  size_t floats = 0;
  auto take = [&](size_t count) {
    float* const here = at ? at + floats : nullptr;
    floats += (count + 3) & ~(size_t)3;
    return here;
  };
  const size_t slots = (size_t)2 * pl.W * pl.block_rows, rows = (size_t)p->b * p->c.h_kv * p->R;
  if (pl.split) {
    p->part_o = take(slots * p->c.v);
    p->part_m = take(slots);
    p->part_l = take(slots);
    p->starts = reinterpret_cast<int32_t*>(take((size_t)p->b + 1));
  }
  if (p->scores_out) {
    p->stats = take(rows * 2);
    p->logits = take(rows * (((size_t)p->c.positions() + kPagedTile - 1) / kPagedTile * kPagedTile));
  }
  return floats * sizeof(float);
}

PagedPlan paged_plan(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v, int is_bf16, int with_scores) {
  PagedPlan pl = {};
  const long long R = (long long)n * (h / h_kv), positions = (long long)max_pages * page_size, tiles = (positions + kPagedTile - 1) / kPagedTile;
  pl.mfma = false;
  pl.block_rows = kScalarRows;
  pl.blocks = (int)((R + pl.block_rows - 1) / pl.block_rows);
  const long long units = (long long)b * h_kv * pl.blocks;
  pl.split = tiles > 8;
  pl.W = pl.split ? kPagedWorkgroups : (int)units;
  if (pl.split && units * tiles / kLeastTiles < pl.W) pl.W = (int)(units * tiles / kLeastTiles);
  PagedDecode p = {};
  p.b = b; p.R = (int)R;
  p.c.h_kv = h_kv; p.c.v = v; p.c.page_size = page_size; p.c.max_pages = max_pages;
  p.scores_out = with_scores ? reinterpret_cast<float*>(1) : nullptr;
  pl.bytes = lay_out(&p, pl, nullptr);
  return pl;
}

void paged_workspace(PagedDecode* p, const PagedPlan& pl, void* workspace) { lay_out(p, pl, static_cast<float*>(workspace)); }

hipError_t launch_paged_decode(const PagedDecode& p_in, const PagedPlan& pl, int is_bf16, hipStream_t st) {
  PagedDecode p = p_in;
  const size_t lds = scalar_lds_floats(p.c.k, p.c.v) * sizeof(float);
  if (is_bf16) hipLaunchKernelGGL(paged_scalar_kernel<uint16_t>, dim3((unsigned)pl.W), dim3(kThreads), lds, st, p);
  else hipLaunchKernelGGL(paged_scalar_kernel<float>, dim3((unsigned)pl.W), dim3(kThreads), lds, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long groups = (long long)p.b * p.c.h_kv;
  if (pl.split) {
    const int v4 = p.c.v >> 2, together = 256 / v4;
    const int rows = groups * pl.blocks >= 64 ? (together < pl.block_rows ? together : pl.block_rows) : 1;
    const long long pieces = (pl.block_rows + rows - 1) / rows;
    hipLaunchKernelGGL(paged_merge_kernel, dim3((unsigned)(groups * pl.blocks * pieces)), dim3(256), 0, st, p, rows);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.scores_out) {
    const long long chunks = (p.c.positions() + 255) / 256;
    hipLaunchKernelGGL(paged_scores_kernel, dim3((unsigned)(groups * chunks)), dim3(256), 0, st, p, (int)chunks);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace mqa
