// Attention over paged caches of 8 bits with a scale for each block of positions and head: o = sum_p weights[p] s_V(p) V8[p] of logits scale s_K(p) (q . K8[p]).
//
// The work is cut, merged, and done again in the plain form where infinities and NaN take part, as in paged_decode.hpp.  A workgroup is four waves, wave w has tiles w, w + 4, ... of 32 positions for 16 or
// 32 query rows.  Both products are v_mfma_f32_16x16x32_f16; 8 bits are exact in fp16.
//   logits^T[32 pos x 16 rows] = K_tile . q^T: lane (i, g) has the 16-byte pieces g, g + 4, ... of two K rows, a piece's first eight columns for one product, the others for the next.  q's rows are
//     brought by a power of two to 2^14 at most and taken as two fp16 terms: by the same one where their sizes are much the same, else each by its own, and its logits back.
//   out^T[D cols x 16 rows] += V_tile^T . weights^T: lane (c, g) has 1/16 of the columns of rows 8g .. 8g + 7.
// Weights.  With s_V(p) = 2^E mant and z the logit (log2), u = z + E - ref is what the running maximum M is taken over, row by row, and w = 2^(u - M) the number that multiplies V8 (times mant, where
// a scale is no power of two): a row's largest *contribution* is 2^10 at least, so that two fp16 terms hold every w to 23 bits, and those that are below 2^-12 of it to 2^-35 of
// it, whatever the scales.  The sum is over w 2^-E.  ref follows the tiles' scales (any will do: M goes with it), which keeps u small, and so its rounding.
//
// What bounds it: 64 sequences of 8192 and 32 rows, 136 MB, take 33 us = 4.1 TB/s, vector instructions (the conversions of 8 bits, the softmax) a third of the SIMDs' cycles and the products a sixth;
// 512 sequences of up to 4096 and 64 rows 107 us, vector instructions 42 % and products 26: a SIMD's registers hold two waves, which leave each other's waits open.  Measured and slower: a
// tile at a time for each wave (48.7 and 150), a wave's two tiles as one of 64 positions (50 and 172, by registers that spill; with fewer of them 36 and 121, as the pairs took then), K converted
// where it is multiplied and V's numbers paired after their conversion (35 and 121).
#include "paged_decode.hpp"

namespace mqa {
namespace {

typedef __attribute__((ext_vector_type(1))) uint32_t u32x1;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

__device__ __forceinline__ floatx4 mfma_f16(const u32x4& a, const u32x4& b, const floatx4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// a pair of floats as two fp16 pairs whose sums are the floats to 23 bits
__device__ __forceinline__ uint32_t pack_f16_pair(float a, float b) { return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b}); }
__device__ __forceinline__ void split2(float a, float b, uint32_t (&t)[2]) {
  t[0] = pack_f16_pair(a, b);
  float c, d;                                              // what that leaves, an instruction each (the compiler takes two)
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(c) : "v"(t[0]), "v"(a));
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(d) : "v"(t[0]), "v"(b));
  t[1] = pack_f16_pair(c, d);
}
// Two bytes each of `biased`, whose bytes are int8 + 128, as fp16: 0x6400 + y is 1024 + y.
__device__ __forceinline__ uint32_t int8_f16(uint32_t biased, uint32_t select) {
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, biased, select)) - f16x2{(_Float16)1152.f, (_Float16)1152.f});
}
__device__ __forceinline__ uint32_t e4m3_f16(uint32_t u, bool upper) {
  return __builtin_bit_cast(uint32_t, upper ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, 1.f, false));
}
// Four values of 8 bits as two fp16 pairs.
template <typename T>
__device__ __forceinline__ void halves(uint32_t u, uint32_t* lo, uint32_t* hi) {
  if constexpr (std::is_same<T, E4M3>::value) {
    *lo = e4m3_f16(u, false);
    *hi = e4m3_f16(u, true);
  } else {
    u ^= 0x80808080u;
    *lo = int8_f16(u, 0x04010400u);
    *hi = int8_f16(u, 0x04030402u);
  }
}
// Values 2 x and 2 x + 1 (`upper`: 2 and 3) of two rows' words, as fp16 pairs of one column each.
template <typename T>
__device__ __forceinline__ void turn2(uint32_t row0, uint32_t row1, bool upper, uint32_t* col0, uint32_t* col1) {
  if constexpr (std::is_same<T, E4M3>::value) {
    const uint32_t pairs = __builtin_amdgcn_perm(row1, row0, upper ? 0x07030602u : 0x05010400u);
    *col0 = e4m3_f16(pairs, false);
    *col1 = e4m3_f16(pairs, true);
  } else {
    const uint32_t pairs = __builtin_amdgcn_perm(row1, row0, upper ? 0x07030602u : 0x05010400u) ^ 0x80808080u;
    *col0 = int8_f16(pairs, 0x04010400u);
    *col1 = int8_f16(pairs, 0x04030402u);
  }
}

template <int D> struct Form8 {
  static constexpr int kPieces = D / 32;                   // products of 32 columns
  static constexpr int kTerms = 2;
  static constexpr int kColumns = D / 16;
  typedef typename std::conditional<D == 256, u32x4, typename std::conditional<D == 128, u32x2, u32x1>::type>::type VRow;
  static __device__ __forceinline__ int column(int i, int j4) { return kColumns * i + 4 * j4; }
};
template <int D> struct Form<E4M3, D> : Form8<D> {};
template <int D> struct Form<Int8, D> : Form8<D> {};

template <int D> struct Tile8 {
  u32x4 kr[2][D / 64];
  typename Form8<D>::VRow vr[8];
};

constexpr float kRoom = 4.f;         // log2 of the largest w over 2^kTop before the maximum is moved; with a mantissa below 2 all stay below 2^15
constexpr float kTop = 10.f;
constexpr int kNear = 16;            // ref is moved for scales that are so many powers of two off
// A row's sum and its maximum go apart by the scales: from 2^-kFar to 2^kFar all numbers that count stay float32's; other scales are the plain form's, unless they are below 2^-kNothing
// and their rows are zeros (which an append gives the smallest scale), and then as good as 2^-kFar.
constexpr int kFar = 50, kNothing = 100;

// Rows of q whose largest numbers are no further than 2^kSameSize apart share a power of two: two fp16 terms then hold a row's numbers to 23 bits, or to 2^-30 of its largest (a row of its own: 2^-38).  Beyond
// 2^kNoSize they are the plain form's.  (64 sequences of 8192, 32 heads: every second row 2^10 smaller 40.9 us, all alike 38.8; 512 of up to 4096, 64 heads 121 and 112; 2^70 smaller, in the plain form,
// 1275 and 6001.)
constexpr int kSameSize = 8, kNoSize = 64;

// Of two tiles' positions, in LDS: K's scale with q's power of two, E - ref, 2^-E, the mantissa.
struct Scales { float f[64], e[64], inv[64], mant[64]; };

template <typename T, int D, int HB, bool EXACT>
struct Rows8 : Rows<T, D, HB, false, EXACT> {
  typedef Rows<T, D, HB, false, EXACT> R;
  using R::acc; using R::m_run; using R::l_run; using R::lim; using R::lim_min;
  static constexpr int NH = 16 * HB, KP = D / 32, KT = 2, NJ = D / 16, QOPS = HB * KP * 64;
  static constexpr int ALL = NH * (D / 8), ITEMS = (ALL + kThreads - 1) / kThreads;

  struct Query { float4 v[ITEMS][2]; };
  static __device__ __forceinline__ void load_q(const PagedDecode& p, const Segment& s, int tid, Query* q) {
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      const int idx = tid + it * kThreads, r = idx / (D / 8), c = idx - r * (D / 8);
      const bool sees = idx < ALL && s.row0 + r < p.R && row_limit(p, s.L, s.row0 + r) > s.begin;      // (what a row that sees nothing here holds is nobody's)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        q->v[it][y] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (sees && (EXACT || 8 * c < p.c.k))
          q->v[it][y] = reinterpret_cast<const float4*>(p.q + row_offset(p, s.i, s.e, s.row0 + r) * (EXACT ? D : p.c.k) + 8 * c)[y];
      }
    }
  }
  // As operands, [term][block of 16 rows][product][lane], all brought down by 2^up, which is returned, so that the largest is 2^13 or more and less than 2^14; a row that is far below that by
  // 2^up back[row] (then *apart is set).  NaN makes NaN of its row's logits; an infinity, and rows too far apart, are the plain form's (*odd).
  static __device__ __forceinline__ int store_q(const PagedDecode& p, int tid, Query& q, u32x4* qs, float* s_most, float* back, int* apart, int* odd) {
    float mine[ITEMS], most = 0.f;
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      mine[it] = 0.f;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float4& v = q.v[it][y];
        v.x *= p.qscale; v.y *= p.qscale; v.z *= p.qscale; v.w *= p.qscale;
        mine[it] = fmaxf(mine[it], fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w))));
      }
      most = fmaxf(most, mine[it]);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor(most, off));
    if ((tid & 63) == 0) s_most[tid >> 6] = most;
    __syncthreads();
    most = fmaxf(fmaxf(s_most[0], s_most[1]), fmaxf(s_most[2], s_most[3]));
    auto exponent = [](float x) { return (int)(__float_as_uint(x) >> 23); };
    const int highest = exponent(most), up = highest - (127 + 13);
    if (highest == 255) *odd = 1;
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      constexpr int W = D / 8;                             // lanes of a row
      const int idx = tid + it * kThreads, r = idx / W, c = idx - r * W;
      const uint64_t some = __ballot(mine[it] > 0.f), large = __ballot(exponent(mine[it]) + kSameSize >= highest);
      auto of_row = [tid](uint64_t lanes) { return (uint32_t)(lanes >> (tid & 63 & ~(W - 1))) & (uint32_t)((1ull << W) - 1); };
      int by = up;
      if (const bool small = of_row(some) && !of_row(large); __any(small)) {
        float here = mine[it];
#pragma unroll
        for (int off = 1; off < W; off <<= 1) here = fmaxf(here, __shfl_xor(here, off));
        if (small) {
          by = exponent(here) - (127 + 13);
          *apart = 1;
          if (up - by > kNoSize) *odd = 1;
        }
      }
      if (idx >= ALL) break;
      if (c == 0) back[r] = ldexpf(1.f, by - up);
      const float x[8] = {q.v[it][0].x, q.v[it][0].y, q.v[it][0].z, q.v[it][0].w, q.v[it][1].x, q.v[it][1].y, q.v[it][1].z, q.v[it][1].w};
      const int slot = ((r >> 4) * KP + 2 * (c >> 3) + (c & 1)) * 64 + (r & 15) + 16 * (c >> 1 & 3);
      u32x4 t[2];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        uint32_t w[2];
        split2(ldexpf(x[2 * y], -by), ldexpf(x[2 * y + 1], -by), w);
        t[0][y] = w[0]; t[1][y] = w[1];
      }
      qs[slot] = t[0];
      qs[QOPS + slot] = t[1];
    }
    return __builtin_amdgcn_readfirstlane(up);
  }

  // q . K of a tile; after(x): the multiplications of product x are under way
  template <typename After>
  static __device__ __forceinline__ void first_product(const Tile8<D>& tl, const u32x4* qs, int lane, floatx4 (&sc)[2][HB], After&& after) {
    constexpr int STEPS = KP * KT, DEEP = 3;               // q of a step (product, term): read while the two before are multiplied
    u32x4 b[DEEP][HB], k[2][2];
    auto read = [&](int n) {
#pragma unroll
      for (int hb = 0; hb < HB; ++hb) b[n % DEEP][hb] = qs[n % KT * QOPS + (hb * KP + n / KT) * 64 + lane];
    };
    auto convert = [&](int x) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          uint32_t lo, hi;
          halves<T>(tl.kr[u][x >> 1][2 * (x & 1) + y], &lo, &hi);
          k[x & 1][u][2 * y] = lo;
          k[x & 1][u][2 * y + 1] = hi;
        }
    };
#pragma unroll
    for (int n = 0; n < DEEP - 1; ++n) read(n);
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) sc[0][hb] = sc[1][hb] = floatx4{0.f, 0.f, 0.f, 0.f};
    convert(0);
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
      if (n + DEEP - 1 < STEPS) read(n + DEEP - 1);
      const int x = n / KT;
      if (n % KT == KT - 1 && x + 1 < KP) convert(x + 1);
#pragma unroll
      for (int hb = 0; hb < HB; ++hb)
#pragma unroll
        for (int u = 0; u < 2; ++u) sc[u][hb] = mfma_f16(k[x & 1][u], b[n % DEEP][hb], sc[u][hb]);
      if (n % KT == KT - 1 && x + 1 < KP) {
#pragma unroll
        for (int z = 0; z < 2 * HB; ++z) {
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x2, 4 / HB, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (n % KT == KT - 1) after(x);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // what multiplies V of a tile (the half-th of its two) from position p0 on; apart, back: as store_q has them; bad: bit e: position p0 + e is not there; mantissas: some scale is no power
  // of two
  __device__ __forceinline__ void weights(int lane, int p0, int half, int apart, const float* back, uint32_t bad, const Scales& scales, bool mantissas, const floatx4 (&sc)[2][HB], float (&w)[HB][8]) {
    const int g = lane >> 4;
    auto eight = [g, half](const float (&from)[64], float (&to)[8]) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float4 y = reinterpret_cast<const float4*>(from)[8 * half + 2 * g + x];
        to[4 * x] = y.x; to[4 * x + 1] = y.y; to[4 * x + 2] = y.z; to[4 * x + 3] = y.w;
      }
    };
    float f[8], e8[8], inv[8];
    eight(scales.f, f);
    eight(scales.e, e8);
    eight(scales.inv, inv);
#pragma unroll
    for (int hb = 0; hb < HB; ++hb)
#pragma unroll
      for (int e = 0; e < 8; ++e) w[hb][e] = fmaf(sc[e >> 2][hb][e & 3], f[e], e8[e]);
    if (bad || p0 + kPagedTile > lim_min) {                // what is not there, or not seen (rows apart: in every tile, so that others have one branch here)
      int first = p0 + 8 * g, row = lane & 15;
      asm volatile("" : "+v"(first), "+v"(row));           // (a branch: few tiles have such positions)
      if (apart)                                           // (what e8 rounds away goes by the product that is not yet brought back, and comes down with it)
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) {
          const float y = back[16 * hb + row];
#pragma unroll
          for (int e = 0; e < 8; ++e) w[hb][e] = fmaf(w[hb][e] - e8[e], y, e8[e]);
        }
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
          if ((bad >> (8 * g + e) & 1) || first + e >= lim[hb]) w[hb][e] = -INFINITY;
    }
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) {
      float mx = fmaxf(fmaxf(fmaxf(w[hb][0], w[hb][1]), fmaxf(w[hb][2], w[hb][3])), fmaxf(fmaxf(w[hb][4], w[hb][5]), fmaxf(w[hb][6], w[hb][7])));
      if (__any(mx > m_run[hb] + (kTop + kRoom))) {        // (m_run: the maximum less kTop)
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mnew = fmaxf(m_run[hb], mx - kTop);
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
        w[hb][e] = __builtin_amdgcn_exp2f(w[hb][e] - mref);
        sum = fmaf(w[hb][e], inv[e], sum);
      }
      l_run[hb] += sum;
    }
    if (mantissas) {
      float mant[8];
      eight(scales.mant, mant);
#pragma unroll
      for (int hb = 0; hb < HB; ++hb)
#pragma unroll
        for (int e = 0; e < 8; ++e) w[hb][e] *= mant[e];
    }
  }
  static __device__ __forceinline__ void split(const float (&w)[HB][8], u32x4 (&wt)[HB][2]) {
#pragma unroll
    for (int hb = 0; hb < HB; ++hb)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        uint32_t x[2];
        split2(w[hb][2 * y], w[hb][2 * y + 1], x);
        wt[hb][0][y] = x[0]; wt[hb][1][y] = x[1];
      }
  }
  // Two of the lane's columns at a time, which are brought into the operand's order while the two before are multiplied.
  __device__ __forceinline__ void second_product(const u32x4 (&wt)[HB][2], const Tile8<D>& tl) {
    u32x4 v[2][2];
    auto turn = [&](int x) {
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        uint32_t a, b;
        turn2<T>(tl.vr[2 * y][x >> 1], tl.vr[2 * y + 1][x >> 1], x & 1, &a, &b);
        v[x & 1][0][y] = a;
        v[x & 1][1][y] = b;
      }
    };
    turn(0);
#pragma unroll
    for (int x = 0; x < NJ / 2; ++x) {
      __builtin_amdgcn_sched_barrier(0);
      if (x + 1 < NJ / 2) turn(x + 1);
#pragma unroll
      for (int term = 0; term < 2; ++term)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int hb = 0; hb < HB; ++hb) acc[hb][2 * x + j] = mfma_f16(v[x & 1][j], wt[hb][term], acc[hb][2 * x + j]);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
};

// Loads that stay in L2: several blocks of rows read the same tiles, neighbours on an XCD at about the same time, and half a row is a load (64 sequences of 8192, 32 rows: non-temporal
// 38.6 us, so 35.2).
// NEAR: pools of less than 4 GiB, whose loads take 32-bit offsets (512 sequences of up to 4096, 64 heads: 122 us, so 118.7; 32 of up to 2048, 8 K/V heads of 64 21.8 and 20.9).
template <typename T, int D, int HB, bool EXACT, bool NEAR>
__global__ __launch_bounds__(kThreads, D > 128 ? 1 : 2)
void scaled_matrix_kernel(PagedDecode p) {
  typedef Rows8<T, D, HB, EXACT> R;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ __align__(16) int s_rows[kWaves][2][64];
  __shared__ __align__(16) Scales s_scales[kWaves][2];
  __shared__ float s_most[kWaves], s_back[R::NH];
  __shared__ int s_odd, s_apart;
  Segment s;
  if (!find_segment<true>(p, &s)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i16 = lane & 15, g = lane >> 4;
  int (&places)[2][64] = s_rows[wave];
  const int32_t* table = p.c.table + (size_t)s.i * p.c.max_pages;
  const unsigned char* Kp = static_cast<const unsigned char*>(p.c.K);
  const unsigned char* Vp = static_cast<const unsigned char*>(p.c.V);
  const int ntiles = (s.end - s.begin + kPagedTile - 1) / kPagedTile;

  // ---- A wave's tiles in pairs (t, t + 4): their loads are on their way while the pair before is multiplied; where their rows are is found two pairs ahead, lane l has position
  // l % 32 of tile l / 32.  (What is past the end is read as the last position, a page that holds nothing as the pool's first row.)
  struct Place { int entry, inside; };
  auto look_up = [&](int t) {
    const int pos = min(s.begin + kPagedTile * (t + kWaves * (lane >> 5)) + (lane & 31), max(s.end - 1, 0));
    const unsigned page = (p.c.page_size & (p.c.page_size - 1)) == 0 ? (unsigned)pos >> __builtin_ctz(p.c.page_size) : (unsigned)pos / (unsigned)p.c.page_size;
    return Place{table[page], pos - (int)page * p.c.page_size};
  };
  Tile8<D> tl[2];
  const bool whole_power = (p.block & (p.block - 1)) == 0;
  const int shift = __builtin_ctz(p.block);
  float ks, vs;                                            // the scales of the lane's position, asked for when its place is known
  auto publish = [&](const Place& x, int buf) -> uint64_t {      // bit e of what is returned: position e of the pair is not there
    const bool there = (unsigned)x.entry < (unsigned)p.c.num_pages;
    const int row = there ? (x.entry * p.c.h_kv + s.e) * p.c.page_size + x.inside : 0;
    places[buf][lane] = row;
    asm volatile("" ::: "memory");
    const unsigned at = whole_power ? (unsigned)row >> shift : (unsigned)row / (unsigned)p.block;
    ks = p.K_scales[at];
    vs = p.V_scales[at];
    return __ballot(!there);
  };
  const int k = EXACT ? D : p.c.k, v = EXACT ? D : p.c.v;
  int k_row[2];
  auto offset = [](int row, int width, int column) {       // of a row's bytes
    if constexpr (NEAR) return (uint32_t)row * (uint32_t)width + (uint32_t)column;
    else return (size_t)row * width + column;
  };
  auto take_k = [&](int buf, int half) {
#pragma unroll
    for (int u = 0; u < 2; ++u) k_row[u] = places[buf][32 * half + 8 * (i16 >> 2) + 4 * u + (i16 & 3)];
  };
  auto load_k = [&](int half, int x) {
    const int piece = EXACT ? g + 4 * x : min(g + 4 * x, k / 16 - 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) tl[half].kr[u][x] = reinterpret_cast<const u32x4*>(Kp + offset(k_row[u], k, 16 * piece))[0];
  };
  auto load_v = [&](int buf, int half) {
    constexpr int C = D / 16;
    int v_row[8];
    *reinterpret_cast<int4*>(v_row) = reinterpret_cast<const int4*>(places[buf])[8 * half + 2 * g];
    *reinterpret_cast<int4*>(v_row + 4) = reinterpret_cast<const int4*>(places[buf])[8 * half + 2 * g + 1];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      tl[half].vr[e] = reinterpret_cast<const typename Form8<D>::VRow*>(Vp + offset(v_row[e], v, C * (EXACT ? i16 : min(i16, v / C - 1))))[0];
  };

  if (tid == 0) s_odd = s_apart = 0;
  Place next = look_up(wave);
  typename R::Query q;                                     // requested before the first tile and converted while that is on its way
  R::load_q(p, s, tid, &q);
  uint64_t bad = publish(next, 0);                         // of the pair that is loaded; of the one after it
  next = look_up(wave + 2 * kWaves);
#pragma unroll
  for (int half = 0; half < 2; ++half)
    if (half == 0 || wave + kWaves < ntiles) {
      take_k(0, half);
#pragma unroll
      for (int x = 0; x < D / 64; ++x) load_k(half, x);
      load_v(0, half);
    }
  u32x4* qs = reinterpret_cast<u32x4*>(smem);
  const int up = R::store_q(p, tid, q, qs, s_most, s_back, &s_apart, &s_odd);
  __syncthreads();
  const int apart = __builtin_amdgcn_readfirstlane(s_apart);

  R rows;
  rows.begin(p, s, s.row0, lane);
  if (apart) rows.lim_min = 0;
  // ---- the scales of the pair that `publish` was last called for, into LDS; m_run goes with ref
  int ref = 0;
  uint64_t nothing = 0;                                    // positions whose V is nothing beside the others'
  bool mantissas = false, far = false, tiny = false;       // tiny: a row that is not nothing after all
  auto put_scales = [&](int buf, uint64_t missing) {
    const bool there = !(missing >> lane & 1);
    const uint32_t bits = there ? __float_as_uint(vs) : 0x3f800000u;
    const bool none = bits < (uint32_t)(127 - kNothing) << 23;                      // (0 and the smallest)
    const int exponent = (int)(bits >> 23) - 127;                                   // (a negative scale's: above all others)
    int e = there && !none ? exponent : ref;
    if (__any(e > ref + kNear || e < ref - kNear)) {
      int most = there && !none ? e : INT32_MIN;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) most = max(most, __shfl_xor(most, off));
      most = __builtin_amdgcn_readfirstlane(most);
#pragma unroll
      for (int hb = 0; hb < HB; ++hb) rows.m_run[hb] -= (float)(most - ref);
      ref = most;
      if (!there || none) e = ref;
    }
    far = far || __any(e < -kFar || e > kFar);
    if (none) e = -kFar;                                   // (zeros: all that is in the sum and hardly anything in the maximum, however much of the weight they have)
    Scales& own = s_scales[wave][buf];
    const float f = there ? ldexpf(ks, up) : 0.f;
    own.f[lane] = fmaf(f * 0x1p32f, 0.f, f);               // (NaN from 2^96 on: a product, of up to 2^31 and this, that came out as -infinity would go unnoticed)
    own.e[lane] = (float)(e - ref);
    own.inv[lane] = ldexpf(1.f, -e);
    const uint32_t mant = none ? 0x3f800000u : (bits & 0x7fffffu) | 0x3f800000u;
    own.mant[lane] = __uint_as_float(mant);
    asm volatile("" ::: "memory");
    nothing = __ballot(none);
    mantissas = __any(mant != 0x3f800000u);
  };
  put_scales(0, bad);
  uint64_t bad_next = publish(next, 1);
  next = look_up(wave + 4 * kWaves);
  int buf = 1;
  for (int t = wave; t < ntiles; t += 2 * kWaves) {
    const uint64_t zeros = bad | nothing;
    const bool mantissas_now = mantissas;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half == 1 && t + kWaves >= ntiles) break;        // (and there is no next pair)
      const int p0 = s.begin + kPagedTile * (t + kWaves * half);
      if (zeros) {
        uint32_t mine = (uint32_t)(zeros >> (32 * half)) >> (8 * g), absent = (uint32_t)(bad >> (32 * half)) >> (8 * g);
        asm volatile("" : "+v"(mine), "+v"(absent));       // (a branch)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (mine >> e & 1) {
            uint32_t bits = 0;
#pragma unroll
            for (int x = 0; x < (D > 64 ? D / 64 : 1); ++x) bits |= tl[half].vr[e][x];
            if (std::is_same<T, E4M3>::value) bits &= 0x7f7f7f7fu;      // (-0)
            tiny = tiny || (bits != 0 && !(absent >> e & 1));
            tl[half].vr[e] = typename Form8<D>::VRow{};
          }
      }
      floatx4 sc[2][HB];
      take_k(buf, half);
      __builtin_amdgcn_s_setprio(1);                       // (before the other wave's softmax; 1 % here)
      R::first_product(tl[half], qs, lane, sc, [&](int x) {
        if (x & 1) load_k(half, x >> 1);
      });
      __builtin_amdgcn_s_setprio(0);
      float w[HB][8];
      rows.weights(lane, p0, half, apart, s_back, (uint32_t)(bad >> (32 * half)), s_scales[wave][buf ^ 1], mantissas_now, sc, w);
      u32x4 wt[HB][2];
      R::split(w, wt);
      if (half == 1 || t + kWaves >= ntiles) put_scales(buf, bad_next);
      __builtin_amdgcn_s_setprio(1);
      rows.second_product(wt, tl[half]);
      __builtin_amdgcn_s_setprio(0);
      load_v(buf, half);
    }
    bad = bad_next;
    buf ^= 1;
    bad_next = publish(next, buf);                         // places of the pair after the next one
    next = look_up(t + 6 * kWaves);
  }

  if (far || tiny || rows.odd()) s_odd = 1;
  __syncthreads();                                         // (and the q operands are read)
  if (s_odd) {
    in_plain_form<T>(p, s, R::NH, smem);
    return;
  }
#pragma unroll
  for (int hb = 0; hb < HB; ++hb) rows.m_run[hb] += (float)ref;      // (in which the waves differ)
  rows.put(reinterpret_cast<float*>(smem), wave, lane);
  __syncthreads();
  R::finish(p, s, s.row0, reinterpret_cast<const float*>(smem), tid);
}

}  // namespace

PagedPlan scaled_plan(int b, int n, int h, int h_kv, int page_size, int max_pages, int k, int v) {
  return paged_plan(b, n, h, h_kv, page_size, max_pages, k, v, 1, 0, true);
}

template <typename T, int D, int HB, bool EXACT>
static hipError_t launch_pools(const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  const size_t rows = (size_t)p.c.num_pages * p.c.h_kv * p.c.page_size, widest = p.c.k > p.c.v ? p.c.k : p.c.v;
  return rows * widest < (size_t)1 << 32 ? launch_form<scaled_matrix_kernel<T, D, HB, EXACT, true>>(Lds<T, D, HB>::alone, p, pl, st)
                                         : launch_form<scaled_matrix_kernel<T, D, HB, EXACT, false>>(Lds<T, D, HB>::alone, p, pl, st);
}
template <typename T, int D, bool EXACT>
static hipError_t launch_rows(const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  return pl.block_rows == 32 ? launch_pools<T, D, 2, EXACT>(p, pl, st) : launch_pools<T, D, 1, EXACT>(p, pl, st);
}
template <typename T>
static hipError_t launch_widths(const PagedDecode& p, const PagedPlan& pl, hipStream_t st) {
  switch (pl.form) {
    case 64: return launch_rows<T, 64, true>(p, pl, st);
    case 128: return launch_rows<T, 128, true>(p, pl, st);
    case -64: return launch_rows<T, 64, false>(p, pl, st);
    case -128: return launch_rows<T, 128, false>(p, pl, st);
    default: return launch_rows<T, 256, false>(p, pl, st);
  }
}

hipError_t launch_scaled_decode(const PagedDecode& p, const PagedPlan& pl, int is_e4m3, hipStream_t st) {
  hipError_t e = launch_list(p, pl, st);
  if (e != hipSuccess) return e;
  e = is_e4m3 ? launch_widths<E4M3>(p, pl, st) : launch_widths<Int8>(p, pl, st);
  return e != hipSuccess ? e : launch_finish(p, st);
}

}  // namespace mqa
