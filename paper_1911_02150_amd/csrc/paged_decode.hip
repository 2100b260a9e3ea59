// Attention of the newest tokens of every sequence over a paged cache.
//
// Per (sequence, K/V head) the R = n * h / h_kv query rows share the K and V rows; row r is query j = r / (h / h_kv), which sees the positions below
// lens - (n - 1 - j):
//   logits[r,p] = scale * sum_c q[r,c] K[p,c];  weights = softmax over p;  o[r,:] = sum_p weights[r,p] V[p,:]
// Positions on pages that hold nothing have weight 0, and a row that sees nothing is 0.
#include "paged.hpp"

#include <type_traits>

namespace mqa {
namespace {

constexpr int kThreads = 256;
constexpr int kScalarRows = 8;            // query rows of a pass of the scalar form

// A run of tiles of one group, for one block of its query rows.
struct Segment {
  int i, e, row0;          // sequence, head, first query row of the block
  int L;                   // the sequence's length
  int begin, end;          // positions
  int piece;               // where its partial states go; -1: the segment is the whole group
};

__device__ __forceinline__ size_t row_offset(const PagedDecode& p, int i, int e, int r) {      // of q and o, in rows
  const int group = p.h / p.c.h_kv;
  return ((size_t)i * p.n + r / group) * p.h + (size_t)e * group + r % group;
}
__device__ __forceinline__ int row_limit(const PagedDecode& p, int L, int r) {                 // the first position that row r does not see
  return max(0, L - (p.n - 1 - r / (p.h / p.c.h_kv)));
}
__device__ __forceinline__ size_t logits_pitch(const PagedDecode& p) { return (size_t)((p.c.positions() + kPagedTile - 1) / kPagedTile) * kPagedTile; }

// What a row's weights are taken from: 2^(logit - x) y.  A row that sees nothing: weights of 0.
__device__ __forceinline__ float2 state_of(float m, float l) { return make_float2(m == -INFINITY ? 0.f : m, l == 0.f ? 0.f : 1.f / l); }

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
      if (s.piece < 0) {
        const float inv = state_of(s_m[j], s_l[j]).y;
        a.x *= inv; a.y *= inv; a.z *= inv; a.w *= inv;
        reinterpret_cast<float4*>(p.o + row_offset(p, s.i, s.e, r0 + j) * v)[tid] = a;
      } else {
        reinterpret_cast<float4*>(p.part_o + ((size_t)s.piece * p.R + r0 + j) * v)[tid] = a;
      }
    }
  if (tid < nr) {
    if (s.piece >= 0) {
      p.part_m[(size_t)s.piece * p.R + r0 + tid] = s_m[tid];
      p.part_l[(size_t)s.piece * p.R + r0 + tid] = s_l[tid];
    } else if (p.stats) {
      p.stats[((size_t)s.i * p.c.h_kv + s.e) * p.R + r0 + tid] = state_of(s_m[tid], s_l[tid]);
    }
  }
}

// ---------------------------------------------------------------- the list of work
__device__ __forceinline__ int tiles_of(const PagedDecode& p, int len) { return (paged_length(p.c, len) + kPagedTile - 1) / kPagedTile; }

// Sum of x over the threads before this one; *all: over all.
template <int THREADS = kThreads>
__device__ __forceinline__ int before_me(int x, int* s_waves, int* all) {
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

constexpr int kComputeUnits = 256, kShares = 768, kSharesOfMany = 512, kLeast = 16, kLongest = 64;

// Tiles of a piece, at most: a whole number for each of the workgroup's four waves.
__device__ __forceinline__ int whole_waves(int tiles) { return max(1, (tiles + 3) >> 2) * 4; }
__device__ __forceinline__ int pieces_of(int tiles, int per) { return max(1, (int)((unsigned)(tiles + per - 1) / (unsigned)per)); }
// Many groups: are they left whole?  total: of all groups
__device__ __forceinline__ bool left_whole(const PagedDecode& p, int longest, int total) {
  return longest <= kLongest && longest * (kComputeUnits / p.blocks) <= total;
}
__device__ __forceinline__ int share_of(const PagedDecode& p, int total) {
  const int shares = p.blocks > 1 ? kSharesOfMany : kShares;
  return max(kLeast, (total + shares - 1) / shares);
}

// Thousands of sequences: what look_for finds from all lengths, found once, by one workgroup: p.work[0].x: pieces of one head of all sequences, and behind it for
// each of them {sequence, pieces before the sequence's, the sequence's, its length}.  Looked for by every workgroup it grows with the square of the sequences: 32768 of up
// to 20 positions, 8 heads, 5912 us, from the list 397; 2048 54 and 33; of 300 to 1200, 32 heads, 4096 389 and 315, 1024 91 and 92, 300 38 and 47 (a launch more).
constexpr int kLookedFor = 1024;         // sequences, at most, without it
constexpr int kListThreads = 1024, kListEach = 8;
__global__ __launch_bounds__(kListThreads)
void paged_list_kernel(PagedDecode p) {
  __shared__ int s_waves[3][kListThreads / 64], s_longest[kListThreads / 64];
  const int tid = threadIdx.x;
  int mine = 0, longest = 0;
  for (int x = tid; x < p.b; x += kListThreads) {
    const int t = tiles_of(p, p.lens[x]);
    mine += t;
    longest = max(longest, t);
  }
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) longest = max(longest, __shfl_xor(longest, off));
  if ((tid & 63) == 0) s_longest[tid >> 6] = longest;
  int total;
  before_me<kListThreads>(mine, s_waves[2], &total);
  total *= p.c.h_kv;
#pragma unroll
  for (int w = 0; w < kListThreads / 64; ++w) longest = max(longest, s_longest[w]);
  const int per = whole_waves(left_whole(p, longest, total) ? longest : share_of(p, total));
  int before = 0;
  for (int base = 0, turn = 0; base < p.b; base += kListThreads * kListEach, turn ^= 1) {
    const int first = base + kListEach * tid;
    int len[kListEach], count[kListEach], sum = 0;
#pragma unroll
    for (int x = 0; x < kListEach; ++x) len[x] = p.lens[min(first + x, p.b - 1)];
#pragma unroll
    for (int x = 0; x < kListEach; ++x) {
      count[x] = first + x < p.b ? pieces_of(tiles_of(p, len[x]), per) : 0;
      sum += count[x];
    }
    int all, at = before + before_me<kListThreads>(sum, s_waves[turn], &all);      // (its places are written again two barriers later)
    before += all;
#pragma unroll
    for (int x = 0; x < kListEach; ++x) {
      const int4 work = make_int4(first + x, at, count[x], len[x]);
      for (const int end = at + count[x]; at < end; ++at) p.work[1 + at] = work;
    }
  }
  if (tid == 0) p.work[0] = make_int4(before, 0, 0, 0);
}

// The sequence that a piece is of, which of the sequence's pieces (`off`), and how many a head has (`c`); false: there is no such piece.  Every workgroup looks at all
// lengths: thread t has sequences t * each up to the next one's.
__device__ __forceinline__ bool look_for(const PagedDecode& p, int piece, Segment* s, int* off, int* c) {
  __shared__ int s_waves[8][kThreads / 64], s_longest[kThreads / 64];
  __shared__ int s_at[4];
  const int tid = threadIdx.x, heads = p.c.h_kv;
  const int each = (p.b + kThreads - 1) / kThreads, from = tid * each, to = min(p.b, from + each);
  const int len = from < to ? p.lens[from] : 0;            // (up to 256 sequences: read once)
  int mine = tiles_of(p, len), longest = mine;
  for (int x = from + 1; x < to; ++x) {
    const int t = tiles_of(p, p.lens[x]);
    mine += t;
    longest = max(longest, t);
  }
  const bool many = p.b * heads * p.blocks >= 2 * kComputeUnits;
  if (many) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) longest = max(longest, __shfl_xor(longest, off));
    if ((tid & 63) == 0) s_longest[tid >> 6] = longest;
  }
  int total;
  before_me(mine, s_waves[0], &total);
  total *= heads;
  // Whole groups where there are two for every compute unit, none long and none
  // more than twice what a workgroup's share would be (512 sequences of up to 1000, 32 heads: 45 us, in shares 56; 64 of up to 2500, 8 K/V heads, which this rule cuts,
  // 75, uncut 84).  Else as many as leave every compute unit one workgroup at most, or else two, if
  // that is not too uneven (64 sequences of 8192, 32 heads: 53 us, in 512 pieces 58; 128 of up to 1024, 64 heads, two to a unit 33, in shares of a 768th 45): up to a
  // quarter over an even share each (48 of 2048, 32 heads 23.1, none over it 27.5; 100 of up to 4000 33.7 and 36.9; 90 of 3000, 8 heads 35.8 and 34.5; half over it:
  // no better, and 128 of up to 1024, 64 heads 37.7 for 33.8); else
  // shares so small that a compute unit has several in turn (512 sequences of up to 4096, 32 heads: 126, in shares of a 512th 137, of a 1536th 133; with several
  // blocks of rows shares of a 512th: 300 of up to 6000, 64 heads 160, of a 768th 166), though
  // not below four tiles a wave (256 of 512, 64 heads: 31, else 42).
  int per = 0, count = 0, before = 0, all = 0, turn = 0;
  auto cut = [&](int tiles) {
    per = whole_waves(tiles);
    count = from < to ? pieces_of(tiles_of(p, len), per) : 0;
    for (int x = from + 1; x < to; ++x) count += pieces_of(tiles_of(p, p.lens[x]), per);
    before = before_me(count, s_waves[++turn], &all);
  };
  bool fits = false;
  if (many) {
    longest = max(max(s_longest[0], s_longest[1]), max(s_longest[2], s_longest[3]));
    fits = left_whole(p, longest, total);
    if (fits) cut(longest);
  }
  for (int most = kComputeUnits; most <= 2 * kComputeUnits; most *= 2) {
    const int units = most / p.blocks;
    if (!fits && p.b * heads <= units)
      for (int x = 8; x <= 10 && !fits; ++x) {
        cut((int)(((long long)total * x + 8 * units - 1) / (8 * units)));
        fits = all * heads <= units;
      }
  }
  if (!fits) cut(share_of(p, total));
  if (piece >= all * heads) return false;
  if (before * heads <= piece && piece < (before + count) * heads) {      // one thread
    int x = from, L = len, mine = pieces_of(tiles_of(p, len), per);
    while (piece >= (before + mine) * heads) {
      before += mine;
      L = p.lens[++x];
      mine = pieces_of(tiles_of(p, L), per);
    }
    s_at[0] = x;
    s_at[1] = piece - before * heads;
    s_at[2] = L;
    s_at[3] = mine;
  }
  __syncthreads();
  s->i = __builtin_amdgcn_readfirstlane(s_at[0]);
  *off = __builtin_amdgcn_readfirstlane(s_at[1]);
  *c = __builtin_amdgcn_readfirstlane(s_at[3]);
  s->L = paged_length(p.c, __builtin_amdgcn_readfirstlane(s_at[2]));
  return true;
}

// This workgroup's segment; false: there is none.
__device__ __forceinline__ bool find_segment(const PagedDecode& p, Segment* s) {
  const int tid = threadIdx.x, heads = p.c.h_kv;
  int piece = blockIdx.x, block = 0;
  if (p.blocks > 1) {                    // (workgroups go to the eight XCDs in turn: a piece's are neighbours on one)
    const unsigned turn = blockIdx.x >> 3;
    block = (int)(turn % (unsigned)p.blocks);
    piece = (int)(turn / (unsigned)p.blocks) * 8 + (int)(blockIdx.x & 7);
  }
  s->row0 = block * p.block_rows;
  if (!p.split) {
    if (piece >= p.b * heads) return false;
    s->i = piece / heads;
    s->e = piece - s->i * heads;
    s->L = paged_length(p.c, p.lens[s->i]);
    s->begin = 0;
    s->end = s->L;
    s->piece = -1;
    return true;
  }
  int off, c;
  if (p.work) {
    if (piece >= p.work[0].x * heads) return false;
    const int4 work = p.work[1 + piece / heads];
    s->i = work.x;
    off = piece - work.y * heads;
    c = work.z;
    s->L = paged_length(p.c, work.w);
  } else if (!look_for(p, piece, s, &off, &c)) {
    return false;
  }
  s->e = heads == 1 ? 0 : off / c;
  const int x = off - s->e * c, t = (s->L + kPagedTile - 1) / kPagedTile;
  s->begin = 0;
  s->end = s->L;
  s->piece = -1;
  if (c > 1) {
    s->begin = (int)((unsigned)(x * t) / (unsigned)c) * kPagedTile;
    s->end = min(s->L, (int)((unsigned)((x + 1) * t) / (unsigned)c) * kPagedTile);
    s->piece = piece;
  }
  if (x == 0 && block == 0 && tid == 0) p.spans[(size_t)s->i * heads + s->e] = make_int2(piece, c);
  return true;
}

// ---------------------------------------------------------------- matrix instructions
// Caches of k = v = D = 64 or 128, and (EXACT = false) of any widths up to D = 64, 128 or 256: pieces past a width are read as its last, against q's zeros
// and into columns that nobody wants.  A workgroup is four waves; wave w has the tiles w, w + 4, ... of a segment, for all rows of the block (16 or 32), and keeps
// their running maximum, sum and outputs; at the end the four states are merged through LDS.  Rows go from memory straight into the operands:
//   logits^T[32 pos x 16 rows] = K_tile . q^T: lane (i, g) = (lane % 16, lane / 16) has 16-byte pieces g, g + 4, ... of two K rows.  Row i of product u is position
//     8 (i / 4) + 4u + i % 4 of the tile, so that lane (row, g) ends up with positions 8g .. 8g + 7: the weights are the second product's operand as they are.
//   out^T[D cols x 16 rows] += V_tile^T . weights^T: lane (c, g) has 1/16 of the columns of rows 8g .. 8g + 7.
// bf16: v_mfma_f32_16x16x32_bf16, q and the weights as three bf16 terms (24 bits: the float32 itself), V transposed 8 x 8 inside the lane.  float32:
// v_mfma_f32_16x16x4_f32.  The rows' places are looked up a tile ahead: a lane has a position's table entry, the wave's 32 rows pass through LDS.
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(8))) uint32_t u32x8;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
constexpr float kSlack = 8.f;        // log2 of the largest weight kept before the running maximum is moved (all rows of a wave together)

__device__ __forceinline__ floatx4 mfma_bf16(const u32x4& a, const u32x4& b, const floatx4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// a pair of floats as three bf16 pairs whose sums are the floats
__device__ __forceinline__ void split3(float a, float b, uint32_t (&t)[3]) {
  t[0] = pack_bf16_pair(a, b);
  a -= __uint_as_float(t[0] << 16);
  b -= __uint_as_float(t[0] & 0xffff0000u);
  t[1] = pack_bf16_pair(a, b);
  t[2] = pack_bf16_pair(a - __uint_as_float(t[1] << 16), b - __uint_as_float(t[1] & 0xffff0000u));
}

template <typename T, int D> struct Form;
template <int D> struct Form<uint16_t, D> {
  static constexpr int kPieces = D / 32;                   // 16-byte pieces of a K row in a lane
  static constexpr int kTerms = 3;
  static constexpr int kColumns = D / 16;                  // columns of a lane
  typedef typename std::conditional<D == 256, u32x8, typename std::conditional<D == 128, u32x4, u32x2>::type>::type VRow;
  static __device__ __forceinline__ int column(int i, int j4) { return kColumns * i + 4 * j4; }      // of the products 4 j4 ..: row i
};
template <int D> struct Form<float, D> {
  static constexpr int kPieces = D / 16;
  static constexpr int kTerms = 1;
  static constexpr int kColumns = D / 16;
  struct VRow { floatx4 x[D / 64]; };
  static __device__ __forceinline__ int column(int i, int j4) { return 64 * j4 + 4 * i; }
};

constexpr int kWaves = 4;            // that share a block of rows
template <typename T, int D, int HB> struct Lds {
  static constexpr size_t q = (size_t)Form<T, D>::kTerms * HB * Form<T, D>::kPieces * 64 * 16;                                   // operands
  static constexpr size_t merge = ((size_t)kWaves * 16 * HB * (D + 4) + 2 * kWaves * 16 * HB) * 4;                             // the waves' states
  static constexpr size_t plain = scalar_lds_floats(D, D) * sizeof(float);
  static constexpr size_t alone = q > merge ? (q > plain ? q : plain) : (merge > plain ? merge : plain);
};

template <typename T, int D> struct Tile {
  u32x4 kr[2][Form<T, D>::kPieces];
  typename Form<T, D>::VRow vr[8];
};
// V as the second product wants it: bf16, transposed (its rows' registers are then free for the next tile's).
template <typename T, int D> struct Turned {};
template <int D> struct Turned<uint16_t, D> { u32x4 a[D / 16]; };

// A wave's rows, 16 HB of a group from row0 on, and what they have seen.
template <typename T, int D, int HB, bool SCORED, bool EXACT>
struct Rows {
  typedef Form<T, D> F;
  static constexpr int NH = 16 * HB, KP = F::kPieces, KT = F::kTerms, NJ = F::kColumns, QOPS = HB * KP * 64;
  static constexpr int EACH = 16 / sizeof(T), ALL = NH * (D / EACH), ITEMS = (ALL + kThreads - 1) / kThreads;      // values of a piece of q; pieces of a thread
  floatx4 acc[HB][NJ];
  float m_run[HB], l_run[HB];
  int lim[HB], lim_min;                // the first position that a lane's row does not see, and the first that not all rows see

  // q: on its way, and (tid: of the 256 threads that share the rows) as operands of the first product, [term][block of 16 rows][piece][lane]
  struct Query { float4 v[ITEMS][EACH / 4]; };
  static __device__ __forceinline__ void load_q(const PagedDecode& p, const Segment& s, int row0, int tid, Query* q) {
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      const int idx = tid + it * kThreads, r = idx / (D / EACH), c = idx - r * (D / EACH);
#pragma unroll
      for (int y = 0; y < EACH / 4; ++y) {
        q->v[it][y] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (idx < ALL && row0 + r < p.R && (EXACT || EACH * c < p.c.k))
          q->v[it][y] = reinterpret_cast<const float4*>(p.q + row_offset(p, s.i, s.e, row0 + r) * (EXACT ? D : p.c.k) + EACH * c)[y];
      }
    }
  }
  static __device__ __forceinline__ void store_q(const PagedDecode& p, int tid, const Query& q, u32x4* qs) {
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      const int idx = tid + it * kThreads, r = idx / (D / EACH), c = idx - r * (D / EACH);
      if (idx >= ALL) break;
      float x[EACH];
#pragma unroll
      for (int y = 0; y < EACH / 4; ++y) {
        const float4 v = q.v[it][y];
        x[4 * y] = v.x * p.qscale; x[4 * y + 1] = v.y * p.qscale; x[4 * y + 2] = v.z * p.qscale; x[4 * y + 3] = v.w * p.qscale;
      }
      const int slot = ((r >> 4) * KP + (c >> 2)) * 64 + (r & 15) + 16 * (c & 3);
      if constexpr (sizeof(T) == 2) {
        u32x4 t[3];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          uint32_t w[3];
          split3(x[2 * y], x[2 * y + 1], w);
          t[0][y] = w[0]; t[1][y] = w[1]; t[2][y] = w[2];
        }
#pragma unroll
        for (int y = 0; y < 3; ++y) qs[y * QOPS + slot] = t[y];
      } else {
        qs[slot] = u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
      }
    }
  }

  __device__ __forceinline__ void begin(const PagedDecode& p, const Segment& s, int row0, int lane) {
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) {
      m_run[hb] = -INFINITY;
      l_run[hb] = 0.f;
      lim[hb] = row_limit(p, s.L, min(row0 + 16 * hb + (lane & 15), p.R - 1));
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[hb][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    lim_min = row_limit(p, s.L, min(row0, p.R - 1));
  }

  // logits of a tile, from its K rows; after(x): the multiplications of piece x are under way and its registers free
  template <typename After>
  static __device__ __forceinline__ void first_product(const Tile<T, D>& tl, const u32x4* qs, int lane, floatx4 (&sc)[2][HB], After&& after) {
    constexpr int STEPS = KP * KT, DEEP = 3;               // q of a step (piece, term): read while the two before are multiplied
    u32x4 b[DEEP][HB];
    auto read = [&](int n) {
#pragma unroll
      for (int hb = 0; hb < HB; ++hb) b[n % DEEP][hb] = qs[n % KT * QOPS + (hb * KP + n / KT) * 64 + lane];
    };
#pragma unroll
    for (int n = 0; n < DEEP - 1; ++n) read(n);
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) sc[0][hb] = sc[1][hb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
      if (n + DEEP - 1 < STEPS) read(n + DEEP - 1);
      __builtin_amdgcn_sched_barrier(0);
      const int x = n / KT;
#pragma unroll
      for (int y = 0; y < (sizeof(T) == 2 ? 1 : 4); ++y)
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if constexpr (sizeof(T) == 2)
              sc[u][hb] = mfma_bf16(tl.kr[u][x], b[n % DEEP][hb], sc[u][hb]);
            else
              sc[u][hb] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(tl.kr[u][x][y]), __uint_as_float(b[n % DEEP][hb][y]), sc[u][hb], 0, 0, 0);
          }
      if (n % KT == KT - 1) after(x);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // V's part of piece x: NJ / KP of its column groups
  static __device__ __forceinline__ void turn(const Tile<T, D>& tl, int x, Turned<T, D>& v) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int j = x * NJ / KP; j < (x + 1) * NJ / KP; ++j)
#pragma unroll
        for (int y = 0; y < 4; ++y) v.a[j][y] = __builtin_amdgcn_perm(tl.vr[2 * y + 1][j >> 1], tl.vr[2 * y][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
    }
  }

  // the softmax of a tile from position p0 on; bad: bit e: position p0 + e is not there
  __device__ __forceinline__ void weights(const PagedDecode& p, const Segment& s, int row0, int lane, int p0, uint32_t bad, floatx4 (&sc)[2][HB], float (&w)[HB][8]) {
    const int i16 = lane & 15, g = lane >> 4;
    if (bad || p0 + kPagedTile > lim_min) {    // what is not there, or not seen
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
          if ((bad >> (8 * g + e) & 1) || p0 + 8 * g + e >= lim[hb]) sc[e >> 2][hb][e & 3] = -INFINITY;
    }
    if constexpr (SCORED) {
      const size_t pitch = logits_pitch(p);
#pragma unroll
      for (int hb = 0; hb < HB; ++hb)
        if (row0 + 16 * hb + i16 < p.R) {
          float* at = p.logits + (((size_t)s.i * p.c.h_kv + s.e) * p.R + row0 + 16 * hb + i16) * pitch + p0 + 8 * g;
          reinterpret_cast<floatx4*>(at)[0] = sc[0][hb];
          reinterpret_cast<floatx4*>(at)[1] = sc[1][hb];
        }
    }
    // the running maximum is moved when a row's has grown by more than kSlack (any reference will do for the sums)
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) {
      float mx = fmaxf(fmaxf(fmaxf(sc[0][hb][0], sc[0][hb][1]), fmaxf(sc[0][hb][2], sc[0][hb][3])),
                       fmaxf(fmaxf(sc[1][hb][0], sc[1][hb][1]), fmaxf(sc[1][hb][2], sc[1][hb][3])));
      if (__any(mx > m_run[hb] + kSlack)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mnew = fmaxf(m_run[hb], mx);
        const float alpha = __builtin_amdgcn_exp2f(m_run[hb] - (mnew == -INFINITY ? 0.f : mnew));
        l_run[hb] *= alpha;
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[hb][j] *= alpha;
        m_run[hb] = mnew;
      }
      const float mref = m_run[hb] == -INFINITY ? 0.f : m_run[hb];
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[hb][e] = __builtin_amdgcn_exp2f(sc[e >> 2][hb][e & 3] - mref);
        sum += w[hb][e];
      }
      l_run[hb] += sum;
    }
  }
  // after(e): the registers of V row e are free
  template <typename After>
  __device__ __forceinline__ void second_product(const float (&w)[HB][8], const Tile<T, D>& tl, const Turned<T, D>& v, After&& after) {
    if constexpr (sizeof(T) == 2) {
      u32x4 wt[HB][3];
#pragma unroll
      for (int hb = 0; hb < HB; ++hb)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          uint32_t x[3];
          split3(w[hb][2 * y], w[hb][2 * y + 1], x);
          wt[hb][0][y] = x[0]; wt[hb][1][y] = x[1]; wt[hb][2][y] = x[2];
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
#pragma unroll
        for (int term = 0; term < 3; ++term)
#pragma unroll
          for (int hb = 0; hb < HB; ++hb) acc[hb][j] = mfma_bf16(v.a[j], wt[hb][term], acc[hb][j]);
#pragma unroll
        for (int e = 8 * j / NJ; e < 8 * (j + 1) / NJ; ++e) after(e);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int hb = 0; hb < HB; ++hb)
            acc[hb][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(tl.vr[e].x[j >> 2][j & 3], w[hb][e], acc[hb][j], 0, 0, 0);
        after(e);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  // A weight of 0 times an infinity, or one term of a product against another, is NaN: such a segment is done again in the plain form, which multiplies what is seen only.
  __device__ __forceinline__ bool odd() const {
    float x = 0.f;
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) {
      x += 0.f * l_run[hb];
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) x += 0.f * acc[hb][j][r];
    }
    return x != x;
  }

  // The four waves' states in one (all 256 threads that share the rows; `lds` is theirs), and where it goes.
  static constexpr int PITCH = D + 4;
  __device__ __forceinline__ void put(float* lds, int wave, int lane) const {
    const int i16 = lane & 15, g = lane >> 4;
    float *sm = lds + kWaves * NH * PITCH, *sl = sm + kWaves * NH;
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) {
      float* row = lds + ((size_t)wave * NH + 16 * hb + i16) * PITCH;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j4 = 0; j4 < NJ / 4; ++j4)
          *reinterpret_cast<float4*>(row + F::column(4 * g + r, j4)) =
              make_float4(acc[hb][4 * j4][r], acc[hb][4 * j4 + 1][r], acc[hb][4 * j4 + 2][r], acc[hb][4 * j4 + 3][r]);
      float l = l_run[hb];                                 // the four lanes of a row share its maximum and have a part of its sum each
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (g == 0) {
        sm[(16 * hb + i16) * kWaves + wave] = m_run[hb];
        sl[(16 * hb + i16) * kWaves + wave] = l;
      }
    }
  }
  static __device__ __forceinline__ void finish(const PagedDecode& p, const Segment& s, int row0, const float* lds, int tid) {
    const float *sm = lds + kWaves * NH * PITCH, *sl = sm + kWaves * NH;
    const int v = EXACT ? D : p.c.v;
    for (int idx = tid; idx < NH * (D / 4); idx += kThreads) {
      const int r = idx / (D / 4), c4 = idx - r * (D / 4);
      if (row0 + r >= p.R) break;
      if (!EXACT && 4 * c4 >= v) continue;
      const float4 m4 = reinterpret_cast<const float4*>(sm)[r], l4 = reinterpret_cast<const float4*>(sl)[r];
      const float ms[4] = {m4.x, m4.y, m4.z, m4.w}, ls[4] = {l4.x, l4.y, l4.z, l4.w};
      const float M = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3])), ref = M == -INFINITY ? 0.f : M;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.f;
#pragma unroll
      for (int x = 0; x < kWaves; ++x) {
        const float f = __builtin_amdgcn_exp2f(ms[x] - ref);
        const float4 o = reinterpret_cast<const float4*>(lds + ((size_t)x * NH + r) * PITCH)[c4];
        a.x += f * o.x; a.y += f * o.y; a.z += f * o.z; a.w += f * o.w;
        l += f * ls[x];
      }
      if (s.piece < 0) {
        const float2 state = state_of(M, l);
        a.x *= state.y; a.y *= state.y; a.z *= state.y; a.w *= state.y;
        reinterpret_cast<float4*>(p.o + row_offset(p, s.i, s.e, row0 + r) * v)[c4] = a;
        if (p.stats && c4 == 0) p.stats[((size_t)s.i * p.c.h_kv + s.e) * p.R + row0 + r] = state;
      } else {
        const size_t at = (size_t)s.piece * p.R + row0 + r;
        reinterpret_cast<float4*>(p.part_o + at * v)[c4] = a;
        if (c4 == 0) {
          p.part_m[at] = M;
          p.part_l[at] = l;
        }
      }
    }
  }
};

template <typename T>
__device__ __forceinline__ void in_plain_form(const PagedDecode& p, const Segment& s, int rows, unsigned char* smem) {
  for (int r0 = s.row0; r0 < min(p.R, s.row0 + rows); r0 += kScalarRows) scalar_segment<T>(p, s, r0, min(p.R - r0, kScalarRows), reinterpret_cast<float*>(smem));
}

// CACHED: several blocks of rows read the same tiles, neighbours on an XCD at about the same time: from memory once and else from L2.  (64 heads of 512
// sequences of up to 4096, back to back: 190 us.  When that took 185, two teams of four waves in a workgroup 207: a workgroup to a compute unit, whose start and end nothing covers; that with
// the tiles in LDS 300; all 64 rows in a wave, two tiles on their way, 260.)
template <typename T, int D, int HB, bool SCORED, bool CACHED, bool EXACT>
__global__ __launch_bounds__(kThreads, D > 128 ? 1 : 2)
void paged_matrix_kernel(PagedDecode p) {
  typedef Rows<T, D, HB, SCORED, EXACT> R;
  typedef Form<T, D> F;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ __align__(16) int s_rows[kWaves][2][32];
  __shared__ int s_odd;
  Segment s;
  if (!find_segment(p, &s)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i16 = lane & 15, g = lane >> 4;
  int (&places)[2][32] = s_rows[wave];
  const int32_t* table = p.c.table + (size_t)s.i * p.c.max_pages;
  const unsigned char* Kp = static_cast<const unsigned char*>(p.c.K);
  const unsigned char* Vp = static_cast<const unsigned char*>(p.c.V);
  const int ntiles = (s.end - s.begin + kPagedTile - 1) / kPagedTile;

  // ---- where a tile's rows are: a lane asks for position lane % 32's.  (What is past the end is read as the last position, which no row sees twice and which holds
  // what the caller wrote; a page that holds nothing as the pool's first row: without branches around them the loads stay in order, and a wait is for those that
  // are needed.)
  struct Place { int entry, inside; };
  auto look_up = [&](int t) {
    const int pos = min(s.begin + kPagedTile * t + (lane & 31), max(s.end - 1, 0));
    const unsigned page = (unsigned)pos / (unsigned)p.c.page_size;
    return Place{table[page], pos - (int)page * p.c.page_size};
  };
  Tile<T, D> tl;
  int k_row[2], v_row[8];                                  // of the tile that is loaded next
  auto publish = [&](const Place& x, int buf) -> uint32_t {      // bit e of what is returned: position e of the tile is not there
    const bool there = (unsigned)x.entry < (unsigned)p.c.num_pages;
    places[buf][lane & 31] = there ? (x.entry * p.c.h_kv + s.e) * p.c.page_size + x.inside : 0;
    asm volatile("" ::: "memory");
    return (uint32_t)__ballot(!there);
  };
  auto take = [&](int buf) {
#pragma unroll
    for (int u = 0; u < 2; ++u) k_row[u] = places[buf][8 * (i16 >> 2) + 4 * u + (i16 & 3)];
    *reinterpret_cast<int4*>(v_row) = reinterpret_cast<const int4*>(places[buf])[2 * g];
    *reinterpret_cast<int4*>(v_row + 4) = reinterpret_cast<const int4*>(places[buf])[2 * g + 1];
  };
  auto read = [](const auto* at) {
    if constexpr (CACHED) return *at;
    else return __builtin_nontemporal_load(at);
  };
  const int k = EXACT ? D : p.c.k, v = EXACT ? D : p.c.v;
  auto load_k = [&](int x) {
    const int piece = EXACT ? g + 4 * x : min(g + 4 * x, k / R::EACH - 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) tl.kr[u][x] = read(reinterpret_cast<const u32x4*>(Kp + (size_t)k_row[u] * (k * sizeof(T))) + piece);
  };
  auto load_v = [&](int e) {
    const unsigned char* src = Vp + (size_t)v_row[e] * (v * sizeof(T));
    if constexpr (sizeof(T) == 2) {
      constexpr int C = F::kColumns;
      if constexpr (EXACT || C <= 8) {
        tl.vr[e] = read(reinterpret_cast<const typename F::VRow*>(src) + (EXACT ? i16 : min(i16, v / C - 1)));
      } else {                                             // 16 columns: two pieces
        const u32x4* at = reinterpret_cast<const u32x4*>(src);
        const u32x4 lo = read(at + min(2 * i16, v / 8 - 1)), hi = read(at + min(2 * i16 + 1, v / 8 - 1));
        tl.vr[e] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    } else {
#pragma unroll
      for (int x = 0; x < D / 64; ++x) tl.vr[e].x[x] = read(reinterpret_cast<const floatx4*>(src) + (EXACT ? 16 * x + i16 : min(16 * x + i16, v / 4 - 1)));
    }
  };

  if (tid == 0) s_odd = 0;
  Place next = look_up(wave);
  typename R::Query q;                                     // requested before the first tile and converted while that is on its way
  R::load_q(p, s, s.row0, tid, &q);
  uint32_t bad = publish(next, 0);                         // of the tile that is loaded; of the one after it
  next = look_up(wave + kWaves);
  take(0);
#pragma unroll
  for (int x = 0; x < F::kPieces; ++x) load_k(x);
#pragma unroll
  for (int e = 0; e < 8; ++e) load_v(e);
  u32x4* qs = reinterpret_cast<u32x4*>(smem);
  R::store_q(p, tid, q, qs);
  __syncthreads();

  R rows;
  rows.begin(p, s, s.row0, lane);
  uint32_t bad_next = publish(next, 1);
  next = look_up(wave + 2 * kWaves);
  take(1);
  int buf = 1;
  for (int t = wave; t < ntiles; t += kWaves) {
    const int p0 = s.begin + kPagedTile * t;
    const uint32_t now = bad;
    if (now) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (now >> (8 * g + e) & 1) tl.vr[e] = typename F::VRow{};
    }
    floatx4 sc[2][HB];
    Turned<T, D> turned;
    R::first_product(tl, qs, lane, sc, [&](int x) {
      load_k(x);
      R::turn(tl, x, turned);
    });
    bad = bad_next;
    buf ^= 1;
    bad_next = publish(next, buf);                         // places of the tile after the next one
    next = look_up(t + 3 * kWaves);
    float w[HB][8];
    rows.weights(p, s, s.row0, lane, p0, now, sc, w);
    rows.second_product(w, tl, turned, load_v);
    take(buf);
  }

  if (rows.odd()) s_odd = 1;
  __syncthreads();                                         // (and the q operands are read)
  if (s_odd) {
    in_plain_form<T>(p, s, R::NH, smem);
    return;
  }
  rows.put(reinterpret_cast<float*>(smem), wave, lane);
  __syncthreads();
  R::finish(p, s, s.row0, reinterpret_cast<const float*>(smem), tid);
}

// ---------------------------------------------------------------- merge
// With (m_s, l_s, acc_s) the partial states: M = max m_s, l = sum l_s 2^(m_s - M), o = sum acc_s 2^(m_s - M) / l.  A workgroup has `rows` rows of a group,
// thread = (four columns, row, every `parts`-th piece).
__device__ __forceinline__ void merge_rows(const PagedDecode& p, int g, int row0, int rows, float (&s_m)[256], float (&s_l)[256], float4 (&s_a)[256]) {
  const int2 span = p.spans[g];
  if (span.y == 1) return;                               // finished by its piece
  const int v4 = p.c.v >> 2, tid = threadIdx.x, parts = 256 / (v4 * rows);
  const int line = tid / v4, c4 = tid - line * v4, part = line / rows, r = row0 + line - part * rows;
  const bool mine = part < parts && r < p.R;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  float M = -INFINITY, l = 0.f;
  const int count = span.y;
  if (mine)
    for (int x0 = part; x0 < count; x0 += 4 * parts) {
      float pm[4], pl[4];
      float4 po[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const size_t at = ((size_t)span.x + min(x0 + x * parts, count - 1)) * p.R + r;
        pm[x] = p.part_m[at];
        pl[x] = p.part_l[at];
        po[x] = reinterpret_cast<const float4*>(p.part_o + at * p.c.v)[c4];
      }
      float Mn = M;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (x0 + x * parts < count) Mn = fmaxf(Mn, pm[x]);
      const float ref = Mn == -INFINITY ? 0.f : Mn, f0 = __builtin_amdgcn_exp2f(M - ref);
      a.x *= f0; a.y *= f0; a.z *= f0; a.w *= f0;
      l *= f0;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (x0 + x * parts < count) {
          const float f = __builtin_amdgcn_exp2f(pm[x] - ref);
          a.x += f * po[x].x; a.y += f * po[x].y; a.z += f * po[x].z; a.w += f * po[x].w;
          l += f * pl[x];
        }
      M = Mn;
    }
  if (parts > 1) {
    s_m[tid] = M;
    s_l[tid] = l;
    s_a[tid] = a;
    __syncthreads();
    if (part != 0) return;
    const int all = v4 * rows;
    for (int x = 1; x < parts; ++x) M = fmaxf(M, s_m[x * all + tid]);
    const float ref = M == -INFINITY ? 0.f : M;
    a = make_float4(0.f, 0.f, 0.f, 0.f);
    l = 0.f;
    for (int x = 0; x < parts; ++x) {
      const float f = __builtin_amdgcn_exp2f(s_m[x * all + tid] - ref);
      const float4 o = s_a[x * all + tid];
      a.x += f * o.x; a.y += f * o.y; a.z += f * o.z; a.w += f * o.w;
      l += f * s_l[x * all + tid];
    }
  }
  if (!mine) return;
  const float inv = state_of(M, l).y;
  a.x *= inv; a.y *= inv; a.z *= inv; a.w *= inv;
  const int heads = p.c.h_kv, i = g / heads;
  reinterpret_cast<float4*>(p.o + row_offset(p, i, g - i * heads, r) * p.c.v)[c4] = a;
}

// scores_out[p] = (p is older than this step's tokens ? scores_in[p] : 0) + sum over the rows of their weights at p.  A workgroup has 256 positions, a wave every
// fourth row of them (1024 positions, all rows of a thread's four: 32 x 32 rows x 8192 positions 10.2 us, so 9.1).
constexpr int kScored = 256;
__device__ __forceinline__ void add_scores(const PagedDecode& p, int g, int chunk, float2* s_state, floatx4 (&s_sum)[4][64]) {
  const int tid = threadIdx.x, i = g / p.c.h_kv, L = paged_length(p.c, p.lens[i]);
  if (chunk * kScored >= L) return;
  int2 span = make_int2(0, 1);
  if (p.split) span = p.spans[g];
  if (span.y == 1) {
    for (int r = tid; r < p.R; r += 256) s_state[r] = p.stats[(size_t)g * p.R + r];
  } else {                                               // the rows' states from their parts': `parts` neighbouring threads a row
    int parts = 64;
    while (parts > 1 && parts * p.R > 256) parts >>= 1;
    const int count = span.y, part = tid % parts;
    for (int r = tid / parts; r < p.R; r += 256 / parts) {
      float M = -INFINITY, l = 0.f;
      for (int x = part; x < count; x += parts) {
        const size_t at = ((size_t)span.x + x) * p.R + r;
        const float m = p.part_m[at], Mn = fmaxf(M, m), ref = Mn == -INFINITY ? 0.f : Mn;
        l = l * __builtin_amdgcn_exp2f(M - ref) + p.part_l[at] * __builtin_amdgcn_exp2f(m - ref);
        M = Mn;
      }
      for (int off = 1; off < parts; off <<= 1) {
        const float m = __shfl_xor(M, off), y = __shfl_xor(l, off), Mn = fmaxf(M, m), ref = Mn == -INFINITY ? 0.f : Mn;
        l = l * __builtin_amdgcn_exp2f(M - ref) + y * __builtin_amdgcn_exp2f(m - ref);
        M = Mn;
      }
      if (part == 0) s_state[r] = state_of(M, l);
    }
  }
  __syncthreads();
  const int lane = tid & 63, wave = tid >> 6, pos = chunk * kScored + 4 * lane;
  const size_t pitch = logits_pitch(p);
  // (the logits of a tile are there whole: past the length, for its last 31 positions, -inf)
  const float* z = p.logits + (size_t)g * p.R * pitch + min(pos, (L - 1) / kPagedTile * kPagedTile + kPagedTile - 4);
  floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int r = wave; r < p.R; r += 4) {
    const floatx4 x = __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(z + r * pitch));
    const float2 state = s_state[r];
#pragma unroll
    for (int y = 0; y < 4; ++y) sum[y] += __builtin_amdgcn_exp2f(x[y] - state.x) * state.y;
  }
  // A row that is NaN makes NaN of 2^-inf as well: a sum that came out so is taken again, over the rows that see the position.
#pragma unroll
  for (int y = 0; y < 4; ++y)
    if (sum[y] != sum[y] && pos + y < L) {
      float again = 0.f;
      if (paged_row(p.c, p.c.table + (size_t)i * p.c.max_pages, 0, pos + y) >= 0)
        for (int r = wave; r < p.R; r += 4)
          if (pos + y < row_limit(p, L, r)) again += __builtin_amdgcn_exp2f(z[r * pitch + y] - s_state[r].x) * s_state[r].y;
      sum[y] = again;
    }
  s_sum[wave][lane] = sum;
  __syncthreads();
  const int mine = chunk * kScored + tid;
  if (mine >= L) return;
  const float* at0 = reinterpret_cast<const float*>(s_sum);
  const float here = (at0[tid] + at0[256 + tid]) + (at0[512 + tid] + at0[768 + tid]);
  const size_t at = (size_t)g * p.c.positions() + mine;
  p.scores_out[at] = (p.scores_in && mine < L - p.n ? p.scores_in[at] : 0.f) + here;
}

// Workgroups of merge_rows, `pieces` a group, then of add_scores, `chunks` a group.
__global__ __launch_bounds__(256)
void paged_finish_kernel(PagedDecode p, int rows, int pieces, int chunks) {
  __shared__ union Shared {
    struct { float m[256], l[256]; float4 a[256]; } merge;
    struct { float2 state[kPagedMaxRows]; floatx4 sum[4][64]; } scores;
    __device__ Shared() {}
  } s;
  const unsigned merging = (unsigned)pieces * p.b * p.c.h_kv;
  if (blockIdx.x < merging) {
    const int g = (int)(blockIdx.x / (unsigned)pieces);
    merge_rows(p, g, ((int)blockIdx.x - g * pieces) * rows, rows, s.merge.m, s.merge.l, s.merge.a);
  } else {
    const int g = (int)((blockIdx.x - merging) / (unsigned)chunks);
    add_scores(p, g, (int)(blockIdx.x - merging) - g * chunks, s.scores.state, s.scores.sum);
  }
}

}  // namespace

// The parts of a call's workspace, each on 16 bytes; their size in all.
static size_t lay_out(PagedDecode* p, const PagedPlan& pl, float* at) {
  size_t floats = 0;
  auto take = [&](size_t count) {
    float* const here = at ? at + floats : nullptr;
    floats += (count + 3) & ~(size_t)3;
    return here;
  };
  const size_t states = (size_t)pl.pieces * p->R, groups = (size_t)p->b * p->c.h_kv;
  if (pl.split) {
    p->part_o = take(states * p->c.v);
    p->part_m = take(states);
    p->part_l = take(states);
    p->spans = reinterpret_cast<int2*>(take(groups * 2));
    if (pl.listed) p->work = reinterpret_cast<int4*>(take(4 * ((size_t)p->b + kShares + 1)));
  }
  if (p->scores_out) {
    p->stats = reinterpret_cast<float2*>(take(groups * p->R * 2));
    p->logits = take(groups * p->R * (((size_t)p->c.positions() + kPagedTile - 1) / kPagedTile * kPagedTile));
  }
  return floats * sizeof(float);
}

PagedPlan paged_plan(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v, int is_bf16, int with_scores) {
  PagedPlan pl = {};
  const long long R = (long long)n * (h / h_kv), positions = (long long)max_pages * page_size, tiles = (positions + kPagedTile - 1) / kPagedTile;
  const int wide = k > v ? k : v;
  pl.form = k == v && (k == 64 || k == 128) ? k : wide <= 64 ? -64 : wide <= 128 ? -128 : -256;
  const long long groups = (long long)b * h_kv;
  // 16 query rows to a workgroup where the work is so little that its latency counts, else 32, whose tiles are read half as often: 16 sequences of 2048, 32 heads
  // 15.0 us against 19.1, 48 of them 22.7 and 23.2, 512 of up to 4096 with 64 heads 249 and 190; 8 sequences of 200, 64 heads 7.8 and 11.0; 256 wide, 32 heads, 16
  // sequences of 2048 24.4 and 28.5, 32 of them 32.5 and 32.0.
  // And only where a compute unit can hold them all, two each, three of 64 wide: 200 sequences of up to 100, 64 heads, 15.5 and 13.5; 64 wide 150 of 40 7.4 and 8.7.
  // (float32 rows of more than 64: 32 query rows do not fit a wave's registers beside a tile.)
  const bool little = groups * tiles * R * (pl.form == -256 ? 4 : 2) <= 3 << 16 && groups * ((R + 15) / 16) <= (wide <= 64 ? 3 : 2) * kComputeUnits;
  pl.block_rows = R <= 16 || little || (!is_bf16 && wide > 64) ? 16 : 32;
  pl.blocks = (int)((R + pl.block_rows - 1) / pl.block_rows);
  // One launch, a workgroup to a group, where cutting and merging would take longer (8 heads, 32 sequences of 500: 10.3 us, in pieces 12.0; of 640 12.9 and 12.3, of 800 15.7
  // and 12.6; one of 500 9.2 and 11.1, of 800 12.0 and 11.1; float32, one of 380 13.6 both, of 500 15.9 and 13.6), and to greater lengths where there is one for
  // every compute unit (256 of up to 1000, 32 heads: 25, in pieces 32).
  const bool heavy = wide > 128 || (!is_bf16 && wide > 64);
  pl.split = tiles > (groups * pl.blocks >= kComputeUnits ? 32 : heavy ? 12 : 16);
  pl.listed = pl.split && b > kLookedFor;
  const long long least = groups * ((tiles + 3) / 4), most = groups + kShares;      // (pieces of four tiles; a last, shorter one in every group)
  pl.pieces = (int)(!pl.split ? groups : least < most ? least : most);
  PagedDecode p = {};
  p.b = b; p.R = (int)R;
  p.c.h_kv = h_kv; p.c.v = v; p.c.page_size = page_size; p.c.max_pages = max_pages;
  p.scores_out = with_scores ? reinterpret_cast<float*>(1) : nullptr;
  pl.bytes = lay_out(&p, pl, nullptr);
  return pl;
}

void paged_workspace(PagedDecode* p, const PagedPlan& pl, void* workspace) { lay_out(p, pl, static_cast<float*>(workspace)); }

// More than 64 KiB of LDS has to be asked for, once per device and kernel.
template <void (*kernel)(PagedDecode)>
static hipError_t launch_form(size_t lds, const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  static bool done[64] = {};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) dev = 0;
  if (lds > 60 * 1024 && !done[dev]) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    done[dev] = true;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)(pl.blocks > 1 ? (pl.pieces + 7) / 8 * 8 : pl.pieces) * pl.blocks), dim3(kThreads), lds, st, p);
  return hipGetLastError();
}
template <typename T, int D, int HB, bool CACHED, bool EXACT>
static hipError_t launch_matrix(const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  constexpr size_t lds = Lds<T, D, HB>::alone;
  return p.scores_out ? launch_form<paged_matrix_kernel<T, D, HB, true, CACHED, EXACT>>(lds, p, pl, st)
                      : launch_form<paged_matrix_kernel<T, D, HB, false, CACHED, EXACT>>(lds, p, pl, st);
}
template <typename T, int D, bool EXACT>
static hipError_t launch_rows(const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  constexpr bool narrow = sizeof(T) == 4 && D > 64;             // (then never 32 rows)
  if constexpr (!EXACT) {
    if constexpr (!narrow)
      if (pl.block_rows == 32) return launch_matrix<T, D, 2, true, false>(p, pl, st);
    return launch_matrix<T, D, 1, true, false>(p, pl, st);
  } else if constexpr (narrow) {
    return pl.blocks > 1 ? launch_matrix<T, D, 1, true, true>(p, pl, st) : launch_matrix<T, D, 1, false, true>(p, pl, st);
  } else {
    if (pl.block_rows == 16) return pl.blocks > 1 ? launch_matrix<T, D, 1, true, true>(p, pl, st) : launch_matrix<T, D, 1, false, true>(p, pl, st);
    return pl.blocks > 1 ? launch_matrix<T, D, 2, true, true>(p, pl, st) : launch_matrix<T, D, 2, false, true>(p, pl, st);
  }
}

hipError_t launch_paged_decode(const PagedDecode& p, const PagedPlan& pl, int is_bf16, hipStream_t st) {
  hipError_t e;
  if (pl.listed) {
    hipLaunchKernelGGL(paged_list_kernel, dim3(1), dim3(kListThreads), 0, st, p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  switch (pl.form) {
    case 64: e = is_bf16 ? launch_rows<uint16_t, 64, true>(p, pl, st) : launch_rows<float, 64, true>(p, pl, st); break;
    case 128: e = is_bf16 ? launch_rows<uint16_t, 128, true>(p, pl, st) : launch_rows<float, 128, true>(p, pl, st); break;
    case -64: e = is_bf16 ? launch_rows<uint16_t, 64, false>(p, pl, st) : launch_rows<float, 64, false>(p, pl, st); break;
    case -128: e = is_bf16 ? launch_rows<uint16_t, 128, false>(p, pl, st) : launch_rows<float, 128, false>(p, pl, st); break;
    default: e = is_bf16 ? launch_rows<uint16_t, 256, false>(p, pl, st) : launch_rows<float, 256, false>(p, pl, st); break;
  }
  if (e != hipSuccess) return e;
  const long long groups = (long long)p.b * p.c.h_kv;
  int rows = 1, pieces = 0, chunks = 0;
  if (p.split) {
    // A workgroup to a row, whose pieces its threads share, or as many rows as it has threads for: together where there are rows enough to fill the chip (32 heads of 8192
    // positions: 2 sequences 26.1 us together, 13.9 alone; 16 26.8 and 25.2; 32 35.9 both; 64 56.1 and 58.3).
    const int together = 256 / (p.c.v >> 2);
    rows = groups * p.R >= 1024 ? (together < p.R ? together : p.R) : 1;
    pieces = (p.R + rows - 1) / rows;
  }
  if (p.scores_out) chunks = (p.c.positions() + kScored - 1) / kScored;
  if (pieces + chunks == 0) return hipSuccess;
  hipLaunchKernelGGL(paged_finish_kernel, dim3((unsigned)(groups * (pieces + chunks))), dim3(256), 0, st, p, rows, pieces, chunks);
  return hipGetLastError();
}

}  // namespace mqa
