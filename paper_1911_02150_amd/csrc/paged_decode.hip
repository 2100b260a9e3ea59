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
  long long at = 0, end = 1;
  int i = 0, first = 0;
  if (p.split) {
    const int per = (p.b + kThreads - 1) / kThreads;
    int tiles, mine;
    const int before = tiles_before_me(p, per, s_waves, &tiles, &mine);
    if (blockIdx.x == 0) {                                      // for the merge
      int from = before;
      for (int x = 0; x < per; ++x) {
        const long long seq = (long long)tid * per + x;
        if (seq > p.b) break;
        p.starts[seq] = from;
        if (seq < p.b) from += tiles_of(p, (int)seq);
      }
      if (tid == 0) p.starts[p.b] = tiles;
    }
    const long long total = tiles * units, W = sharing(p, total), w = blockIdx.x;
    if (w >= W || total == 0) return;
    at = w * total / W;
    end = (w + 1) * total / W;
    if (before * units <= at && at < (before + mine) * units) { // one thread: its sequences hold the first tile
      int from = before;
      for (int x = 0; x < per; ++x) {
        const int seq = tid * per + x, t = tiles_of(p, seq);
        if (at < (from + t) * units) {
          s_at[0] = seq;
          s_at[1] = from;
          break;
        }
        from += t;
      }
    }
    __syncthreads();
    i = s_at[0];
    first = s_at[1];
  } else {
    i = (int)(blockIdx.x / units);
  }
  while (at < end) {
    Segment s;
    s.L = paged_length(p.c, p.lens[i]);
    const int t = (s.L + kPagedTile - 1) / kPagedTile;
    int u = (int)(blockIdx.x % units), tile0 = 0, count = t;
    if (p.split) {
      const long long off = at - first * units;
      if (off >= t * units) {                                   // the next sequence
        first += t;
        ++i;
        continue;
      }
      u = (int)(off / t);
      tile0 = (int)(off - (long long)u * t);
      count = (int)min((long long)(t - tile0), end - at);
      at += count;
    } else {
      at = end;
    }
    s.i = i;
    s.e = u / p.blocks;
    s.row0 = (u % p.blocks) * p.block_rows;
    s.begin = tile0 * kPagedTile;
    s.end = min(s.L, (tile0 + count) * kPagedTile);
    s.slot = count == t ? -1 : 2 * (int)blockIdx.x + (tile0 > 0 ? 0 : 1);
    work(s);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads)
void paged_scalar_kernel(PagedDecode p) {
  extern __shared__ __align__(16) float smem[];
  for_segments(p, [&](const Segment& s) { scalar_segment<T>(p, s, s.row0, min(p.R - s.row0, kScalarRows), smem); });
}

// ---------------------------------------------------------------- matrix instructions
// Caches of k = v = D = 64 or 128.  A workgroup is four waves; wave w has the tiles w, w + 4, ... of a segment, for all rows of the block (16 or 32), and keeps
// their running maximum, sum and outputs; at the end the four states are merged through LDS.  Rows go from memory straight into the operands:
//   logits^T[32 pos x 16 rows] = K_tile . q^T: lane (i, g) = (lane % 16, lane / 16) has 16-byte pieces g, g + 4, ... of two K rows.  Row i of product u is position
//     8 (i / 4) + 4u + i % 4 of the tile, so that lane (row, g) ends up with positions 8g .. 8g + 7: the weights are the second product's operand as they are.
//   out^T[D cols x 16 rows] += V_tile^T . weights^T: lane (c, g) has 1/16 of the columns of rows 8g .. 8g + 7.
// bf16: v_mfma_f32_16x16x32_bf16, q and the weights as three bf16 terms (24 bits: the float32 itself), V transposed 8 x 8 inside the lane.  float32:
// v_mfma_f32_16x16x4_f32.  The rows' places are looked up a tile ahead: a lane has a position's table entry, the wave's 32 rows pass through LDS.
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
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
  typedef typename std::conditional<D == 128, u32x4, u32x2>::type VRow;
  static __device__ __forceinline__ int column(int i, int j4) { return kColumns * i + 4 * j4; }      // of the products 4 j4 ..: row i
};
template <int D> struct Form<float, D> {
  static constexpr int kPieces = D / 16;
  static constexpr int kTerms = 1;
  static constexpr int kColumns = D / 16;
  struct VRow { floatx4 x[D / 64]; };
  static __device__ __forceinline__ int column(int i, int j4) { return 64 * j4 + 4 * i; }
};

constexpr int kWaves = 4;
template <typename T, int D, int HB> constexpr size_t matrix_lds_bytes() {
  const size_t q = (size_t)Form<T, D>::kTerms * HB * Form<T, D>::kPieces * 64 * 16, merge = ((size_t)kWaves * 16 * HB * (D + 4) + 2 * kWaves * 16 * HB) * 4;
  const size_t plain = scalar_lds_floats(D, D) * sizeof(float), most = q > merge ? q : merge;
  return most > plain ? most : plain;
}

template <typename T, int D, int HB>
__device__ __forceinline__ void matrix_segment(const PagedDecode& p, const Segment& s, unsigned char* smem, int (*s_rows)[2][32], int* s_bad) {
  typedef Form<T, D> F;
  constexpr int NH = 16 * HB, KP = F::kPieces, KT = F::kTerms, NJ = F::kColumns, QOPS = HB * KP * 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i16 = lane & 15, g = lane >> 4;
  const int32_t* table = p.c.table + (size_t)s.i * p.c.max_pages;
  const unsigned char* Kp = static_cast<const unsigned char*>(p.c.K);
  const unsigned char* Vp = static_cast<const unsigned char*>(p.c.V);
  const int ntiles = (s.end - s.begin + kPagedTile - 1) / kPagedTile;

  // ---- where a tile's rows are
  int entry = -1, inside = 0;
  auto look_up = [&](int t) {                              // lane: position lane % 32
    const int pos = s.begin + kPagedTile * t + (lane & 31);
    entry = -1;
    if (pos < s.end) {
      const unsigned page = (unsigned)pos / (unsigned)p.c.page_size;
      inside = pos - (int)page * p.c.page_size;
      entry = table[page];
    }
  };
  struct Tile { u32x4 kr[2][KP]; typename F::VRow vr[8]; uint32_t bad; } tl;      // bad: bit e: position 8g + e is not there
  auto publish = [&](int buf) {
    const int row = (unsigned)entry < (unsigned)p.c.num_pages ? (entry * p.c.h_kv + s.e) * p.c.page_size + inside : -1;
    if (lane < 32) s_rows[wave][buf][lane] = row;
    asm volatile("" ::: "memory");
  };
  auto load_k = [&](int buf) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int row = s_rows[wave][buf][8 * (i16 >> 2) + 4 * u + (i16 & 3)];
      const u32x4* src = reinterpret_cast<const u32x4*>(Kp + (size_t)max(row, 0) * (D * sizeof(T))) + g;
#pragma unroll
      for (int x = 0; x < KP; ++x) tl.kr[u][x] = __builtin_nontemporal_load(src + 4 * x);
    }
  };
  auto load_v = [&](int buf) {
    int rows[8];
    *reinterpret_cast<int4*>(rows) = reinterpret_cast<const int4*>(s_rows[wave][buf])[2 * g];
    *reinterpret_cast<int4*>(rows + 4) = reinterpret_cast<const int4*>(s_rows[wave][buf])[2 * g + 1];
    tl.bad = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      tl.bad |= (uint32_t)(rows[e] < 0) << e;
      const unsigned char* src = Vp + (size_t)max(rows[e], 0) * (D * sizeof(T));
      if constexpr (sizeof(T) == 2) {
        tl.vr[e] = __builtin_nontemporal_load(reinterpret_cast<const typename F::VRow*>(src) + i16);
      } else {
#pragma unroll
        for (int x = 0; x < D / 64; ++x) tl.vr[e].x[x] = __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(src) + 16 * x + i16);
      }
    }
  };

  __syncthreads();                                         // the LDS of the segment before is read
  if (tid == 0) *s_bad = 0;
  const bool any = wave < ntiles;
  if (any) look_up(wave);

  // ---- q: operands of the first product
  u32x4* qs = reinterpret_cast<u32x4*>(smem);              // [term][block of 16 rows][piece][lane]
  constexpr int EACH = 16 / sizeof(T);                     // values of a piece
  for (int idx = tid; idx < NH * (D / EACH); idx += kThreads) {
    const int r = idx / (D / EACH), c = idx - r * (D / EACH);
    float x[EACH];
#pragma unroll
    for (int y = 0; y < EACH / 4; ++y) {
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (s.row0 + r < p.R) v = reinterpret_cast<const float4*>(p.q + row_offset(p, s.i, s.e, s.row0 + r) * D + EACH * c)[y];
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
  if (any) {
    publish(0);
    if (wave + kWaves < ntiles) look_up(wave + kWaves);
    load_k(0);
    load_v(0);
  }
  __syncthreads();

  floatx4 acc[HB][NJ];
  float m_run[HB], l_run[HB];
  int lim[HB];
#pragma unroll
  for (int hb = 0; hb < HB; ++hb) {
    m_run[hb] = -INFINITY;
    l_run[hb] = 0.f;
    lim[hb] = row_limit(p, s.L, min(s.row0 + 16 * hb + i16, p.R - 1));
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[hb][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const int lim_min = row_limit(p, s.L, s.row0);           // positions from here on are not seen by all rows

  int buf = 0;
  for (int t = wave; t < ntiles; t += kWaves) {
    const int p0 = s.begin + kPagedTile * t;
    const bool more = t + kWaves < ntiles;
    buf ^= 1;
    if (more) {
      publish(buf);
      if (t + 2 * kWaves < ntiles) look_up(t + 2 * kWaves);
    }
    floatx4 sc[2][HB];
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) {
      sc[0][hb] = sc[1][hb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < KP; ++x)
#pragma unroll
        for (int term = 0; term < KT; ++term) {
          const u32x4 b = qs[term * QOPS + (hb * KP + x) * 64 + lane];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if constexpr (sizeof(T) == 2) {
              sc[u][hb] = mfma_bf16(tl.kr[u][x], b, sc[u][hb]);
            } else {
#pragma unroll
              for (int y = 0; y < 4; ++y)
                sc[u][hb] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(tl.kr[u][x][y]), __uint_as_float(b[y]), sc[u][hb], 0, 0, 0);
            }
          }
        }
    }
    const uint32_t bad = tl.bad;
    if (more) load_k(buf);                                 // its registers are free

    if (__any(bad != 0) || p0 + kPagedTile > lim_min) {    // what is not there, or not seen
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool gone = bad >> e & 1;
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
          if (gone || p0 + 8 * g + e >= lim[hb]) sc[e >> 2][hb][e & 3] = -INFINITY;
        if (gone) tl.vr[e] = typename F::VRow{};
      }
    }
    if (p.logits) {
      const size_t pitch = logits_pitch(p);
#pragma unroll
      for (int hb = 0; hb < HB; ++hb)
        if (s.row0 + 16 * hb + i16 < p.R) {
          float* at = p.logits + (((size_t)s.i * p.c.h_kv + s.e) * p.R + s.row0 + 16 * hb + i16) * pitch + p0 + 8 * g;
          reinterpret_cast<floatx4*>(at)[0] = sc[0][hb];
          reinterpret_cast<floatx4*>(at)[1] = sc[1][hb];
        }
    }
    // ---- softmax: the running maximum is moved when a row's has grown by more than kSlack (any reference will do for the sums)
    float w[HB][8];
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) {
      float mx = fmaxf(fmaxf(fmaxf(sc[0][hb][0], sc[0][hb][1]), fmaxf(sc[0][hb][2], sc[0][hb][3])),
                       fmaxf(fmaxf(sc[1][hb][0], sc[1][hb][1]), fmaxf(sc[1][hb][2], sc[1][hb][3])));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mnew = fmaxf(m_run[hb], mx);
      if (__any(mnew > m_run[hb] + kSlack)) {
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
    // ---- outputs
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
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        u32x4 a;
#pragma unroll
        for (int x = 0; x < 4; ++x) a[x] = __builtin_amdgcn_perm(tl.vr[2 * x + 1][j >> 1], tl.vr[2 * x][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int term = 0; term < 3; ++term)
#pragma unroll
          for (int hb = 0; hb < HB; ++hb) acc[hb][j] = mfma_bf16(a, wt[hb][term], acc[hb][j]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int hb = 0; hb < HB; ++hb)
            acc[hb][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(tl.vr[e].x[j >> 2][j & 3], w[hb][e], acc[hb][j], 0, 0, 0);
    }
    if (more) load_v(buf);
  }

  // ---- a weight of 0 times an infinity, or one term of a product against another, is NaN: such a segment is done again in the plain form, which multiplies what is seen only
  float odd = 0.f;
#pragma unroll
  for (int hb = 0; hb < HB; ++hb) {
    odd += 0.f * l_run[hb];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) odd += 0.f * acc[hb][j][r];
  }
  if (odd != odd) *s_bad = 1;
  __syncthreads();                                         // (the q operands are read)
  if (*s_bad) {
    for (int r0 = s.row0; r0 < min(p.R, s.row0 + NH); r0 += kScalarRows)
      scalar_segment<T>(p, s, r0, min(p.R - r0, kScalarRows), reinterpret_cast<float*>(smem));
    return;
  }

  // ---- the four waves' states
  constexpr int PITCH = D + 4;
  float* so = reinterpret_cast<float*>(smem);              // [wave][NH][PITCH]
  float* sm = so + kWaves * NH * PITCH;                    // [NH][wave]
  float* sl = sm + kWaves * NH;
#pragma unroll
  for (int hb = 0; hb < HB; ++hb) {
    float* row = so + ((size_t)wave * NH + 16 * hb + i16) * PITCH;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j4 = 0; j4 < NJ / 4; ++j4)
        *reinterpret_cast<float4*>(row + F::column(4 * g + r, j4)) =
            make_float4(acc[hb][4 * j4][r], acc[hb][4 * j4 + 1][r], acc[hb][4 * j4 + 2][r], acc[hb][4 * j4 + 3][r]);
    float l = l_run[hb];                                   // the four lanes of a row share its maximum and have a part of its sum each
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
      sm[(16 * hb + i16) * kWaves + wave] = m_run[hb];
      sl[(16 * hb + i16) * kWaves + wave] = l;
    }
  }
  __syncthreads();
  for (int idx = tid; idx < NH * (D / 4); idx += kThreads) {
    const int r = idx / (D / 4), c4 = idx - r * (D / 4);
    if (s.row0 + r >= p.R) break;
    const float4 m4 = reinterpret_cast<const float4*>(sm)[r], l4 = reinterpret_cast<const float4*>(sl)[r];
    const float ms[4] = {m4.x, m4.y, m4.z, m4.w}, ls[4] = {l4.x, l4.y, l4.z, l4.w};
    const float M = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3])), ref = M == -INFINITY ? 0.f : M;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const float f = __builtin_amdgcn_exp2f(ms[x] - ref);
      const float4 o = reinterpret_cast<const float4*>(so + ((size_t)x * NH + r) * PITCH)[c4];
      a.x += f * o.x; a.y += f * o.y; a.z += f * o.z; a.w += f * o.w;
      l += f * ls[x];
    }
    if (s.slot < 0) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      a.x *= inv; a.y *= inv; a.z *= inv; a.w *= inv;
      reinterpret_cast<float4*>(p.o + row_offset(p, s.i, s.e, s.row0 + r) * D)[c4] = a;
      if (p.stats && c4 == 0) {
        float* stat = p.stats + (((size_t)s.i * p.c.h_kv + s.e) * p.R + s.row0 + r) * 2;
        stat[0] = ref;
        stat[1] = inv;
      }
    } else {
      const size_t at = (size_t)s.slot * p.block_rows + r;
      reinterpret_cast<float4*>(p.part_o + at * D)[c4] = a;
      if (c4 == 0) {
        p.part_m[at] = M;
        p.part_l[at] = l;
      }
    }
  }
}

template <typename T, int D, int HB>
__global__ __launch_bounds__(kThreads, 2)
void paged_matrix_kernel(PagedDecode p) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  __shared__ __align__(16) int s_rows[kWaves][2][32];
  __shared__ int s_bad;
  for_segments(p, [&](const Segment& s) { matrix_segment<T, D, HB>(p, s, smem_raw, s_rows, &s_bad); });
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
  pl.mfma = k == v && (k == 64 || k == 128);
  pl.block_rows = !pl.mfma ? kScalarRows : R <= 16 ? 16 : 32;
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

template <typename T, int D, int HB>
static hipError_t launch_matrix(const PagedDecode& p, hipStream_t st) {
  constexpr size_t lds = matrix_lds_bytes<T, D, HB>();
  if (lds > 62 * 1024) {      // (of the 64 KiB that need no asking the kernel's own arrays are part) opt in, once per device
    static bool done[64] = {};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) dev = 0;
    if (!done[dev]) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(paged_matrix_kernel<T, D, HB>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
      done[dev] = true;
    }
  }
  hipLaunchKernelGGL((paged_matrix_kernel<T, D, HB>), dim3((unsigned)p.W), dim3(kThreads), lds, st, p);
  return hipGetLastError();
}

hipError_t launch_paged_decode(const PagedDecode& p, const PagedPlan& pl, int is_bf16, hipStream_t st) {
  hipError_t e = hipErrorInvalidValue;
  if (pl.mfma) {
    const bool wide = pl.block_rows == 32;
    if (p.c.k == 128) {
      if (is_bf16) e = wide ? launch_matrix<uint16_t, 128, 2>(p, st) : launch_matrix<uint16_t, 128, 1>(p, st);
      else e = wide ? launch_matrix<float, 128, 2>(p, st) : launch_matrix<float, 128, 1>(p, st);
    } else {
      if (is_bf16) e = wide ? launch_matrix<uint16_t, 64, 2>(p, st) : launch_matrix<uint16_t, 64, 1>(p, st);
      else e = wide ? launch_matrix<float, 64, 2>(p, st) : launch_matrix<float, 64, 1>(p, st);
    }
  } else {
    const size_t lds = scalar_lds_floats(p.c.k, p.c.v) * sizeof(float);
    if (is_bf16) hipLaunchKernelGGL(paged_scalar_kernel<uint16_t>, dim3((unsigned)p.W), dim3(kThreads), lds, st, p);
    else hipLaunchKernelGGL(paged_scalar_kernel<float>, dim3((unsigned)p.W), dim3(kThreads), lds, st, p);
    e = hipGetLastError();
  }
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
