// Attention of a caller's query rows over the paged KV cache (laser_attend).
//
// Row i of a span sits at position pos + i and sees the keys t in [kb, ke) with t <= pos + i (causal)
// and t > pos + i - window (window > 0):
//   s_t = scale q.k_t,  m = max s_t,  l = sum exp(s_t - m),  o = sum exp(s_t - m) v_t / l,
//   lse = m + log l;  nothing seen: o = 0, lse = -inf.
// The keys are taken once, in exp2 units, with a running m and l per row.  m is moved, and what has been summed
// rescaled, when a score exceeds it, and then to kSlack above that score: so it moves rarely, no weight is above 1 (the
// sums stay inside fp32 for V up to its largest divided by the keys), and the largest is at least 2^-8 of 1.
//
// The G query heads of a kv head and the rows of a span are the columns of one matrix: column c is row
// c / G, head kvh G + c % G, so that K and V are read once for all of them.  Matrix-core products, K or V
// as the A operand:
//   S^T[t][c] = K[t][:] . Q[c][:],   O^T[d][c] += V^T[d][t] P^T[t][c];
// the second takes P^T as the first leaves it in its accumulators: which position stands in which slot
// of the contraction is free, as long as V is read in the same order.
// Types: K and V as bf16 (bf16, E4M3 and 8-bit integers are exact in it; an integer row's scale goes
// onto the scores, and onto the weights).  bf16 queries are exact.  Their weights are two bf16 parts in workgroups of
// 16 columns (one or two new tokens, and all rows of an fp32 pool; off by at most 2^-16 of themselves), where the second
// costs about 1% (64 sequences of 3,000-14,000, 8B heads, INT8: 191.7 and 193.2 us; a chunk of 200 rows of an fp32 pool
// 22.7 and 23.8).  In wider ones they are rounded to bf16, each off by at most 2^-8 of itself, as the bf16 output is
// anyway: a second part there takes the time of another product (32 columns, 16 sequences of 1,000-9,000, 30 rows, 102
// and 115 us; tiles, 4,096 rows behind 12,288, 1,040 and 1,363).  With
// fp32 queries and output, queries and weights (and fp32 K and V) are split into three bf16 parts, which hold all 24
// bits.  m, l, O: fp32.
// A key that a row does not see may hold anything: its score is replaced, an integer row's weight too
// (whatever the scale), and where the stored V itself can be infinite or NaN, pages that not every
// column sees whole are looked through and, if one has such a value, taken row by row with the
// unseen positions' V zeroed.
#include <cstddef>

#include "device_common.hpp"
#include "kernels.hpp"

namespace laser {

namespace {

constexpr float kSlack = 8.f;
constexpr float kLn2 = 0.6931471805599453f;

template <class T>
__device__ __forceinline__ T ld_const(const void* p) {  // uniform, through the scalar unit
  return *(const __attribute__((address_space(4))) T*)(uint64_t)p;
}

__device__ __forceinline__ uint32_t pk_bf16(float a, float b) {  // rounded to nearest even
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, b2));
}
// a and b in three truncated bf16 parts each, packed pairwise: 8 + 8 + 8 significand bits.
__device__ __forceinline__ void split3(float a, float b, uint32_t* p) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    p[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
    b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
  }
}

// Parts and infinities.  A product with parts adds 0 x inf = NaN where a number has an infinity opposite whose
// lower parts are zero (as those of 1.0 are), and an infinity's own lower parts are inf - inf.  So only leading parts
// may meet an infinite element, and they give what the number itself gives: inf, -inf or NaN.  Queries are split so
// once; K and V are only looked at closely (finite_parts) where a sum has become infinite or NaN (that look costs calls
// without infinities up to 2%: fp32 rows, bf16 pool, 7B heads, 4 sequences to 14,000 20.3 and 20.8 us, 16 sequences of
// 1,000-9,000, 40 rows, 217 and 221; a chunk of 1,000 rows behind 8,000 356 and 359).
//
// The ones of a pair whose leading part is finite, as a mask.
__device__ __forceinline__ uint32_t finite_bf16(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
}
__device__ __forceinline__ bf16x8 finite_parts(bf16x8 x, bf16x8 lead) {
  u32x4 w = __builtin_bit_cast(u32x4, x), t = __builtin_bit_cast(u32x4, lead);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] &= finite_bf16(t[i]);
  return __builtin_bit_cast(bf16x8, w);
}
// A NaN's leading part is a NaN as well (and not an infinity, where only low bits tell it from one).
__device__ __forceinline__ uint32_t quiet(uint32_t w) { return (w & 0x7fffffffu) > 0x7f800000u ? w | 0x400000u : w; }

// The span of a work item (spans are listed by their first item), read from the argument segment itself: an
// index into an argument would have the compiler copy all of it to scratch.  With one span its fields come in the
// first round of loads.
__device__ __forceinline__ AttendSpan item_span(int n_spans, unsigned item) {
  using Words = const __attribute__((address_space(4))) int;
  Words* sp = (Words*)((const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(AttendArgs, sp));
  constexpr int W = sizeof(AttendSpan) / 4;
  static_assert(sizeof(AttendSpan) == 36 && offsetof(AttendSpan, first) == 32, "read as words");
  auto get = [](Words* p) {
    return AttendSpan{p[0], p[1], p[2], p[3], p[4], p[5], p[6], (unsigned)p[7], (unsigned)p[8]};
  };
  if (n_spans == 1) return get(sp);
  const int lane = threadIdx.x & 63;
  const unsigned first = lane < n_spans ? (unsigned)sp[lane * W + 8] : 0xffffffffu;
  return get(sp + W * __builtin_amdgcn_readfirstlane(__builtin_popcountll(__ballot(first <= item)) - 1));
}

// O / l; zero where no weight is (whatever 0 x V gave, V of seen keys that score -infinity being infinite).
__device__ __forceinline__ f32x4 normed(f32x4 o, float l) {
  const float inv = 1.f / l;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = l == 0.f ? 0.f : o[i] * inv;
  return o;
}

// Four output dims of a row, in the rows' type.
template <class IT>
__device__ __forceinline__ void st_out4(const AttendArgs& a, int row, int head, int d, f32x4 v) {
  const int64_t e = row * a.o_row + head * a.o_head + d;
  if constexpr (std::is_same_v<IT, float>) {
    float* p = (float*)a.o + e;
    if (a.o_vec) {
      *(f32x4*)p = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = v[i];
    }
  } else {
    const u32x2 w = {pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
    uint16_t* p = (uint16_t*)a.o + e;
    if (a.o_vec) {
      *(u32x2*)p = w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
  }
}

// Eight dims of a query row as one operand of each part.
// (flip: sign bits to invert in every element, for the kernels that want a positive scale)
template <class IT, int PARTS>
__device__ __forceinline__ void ld_query8(const AttendArgs& a, int64_t e, bf16x8* out, uint32_t flip = 0) {
  if constexpr (std::is_same_v<IT, bf16_t>) {
    const uint16_t* p = (const uint16_t*)a.q + e;
    u32x4 w;
    if (a.q_vec) {
      w = ld_global<u32x4>(p);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] ^= flip | (flip >> 16);
    out[0] = __builtin_bit_cast(bf16x8, w);
  } else {
    const float* p = (const float*)a.q + e;
    f32x4 x[2];
    if (a.q_vec) {
      x[0] = ld_global<f32x4>(p);
      x[1] = ld_global<f32x4>(p + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i >> 2][i & 3] = p[i];
    }
    u32x4 w[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t s[3];
      split3(__uint_as_float(quiet(__float_as_uint(x[i >> 1][2 * (i & 1)]))),
             __uint_as_float(quiet(__float_as_uint(x[i >> 1][2 * (i & 1) + 1]))), s);
      const uint32_t fin = finite_bf16(s[0]);
#pragma unroll
      for (int k = 0; k < 3; ++k) w[k][i] = (k == 0 ? s[k] : s[k] & fin) ^ (flip | (flip >> 16));
    }
#pragma unroll
    for (int k = 0; k < PARTS; ++k) out[k] = __builtin_bit_cast(bf16x8, w[k]);
  }
}

__device__ __forceinline__ bool odd_bf16(uint32_t w) {  // one of a pair is infinite or NaN
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

}  // namespace

// A piece of a page that other workgroups read as well (SH: it stays in the caches), or none.
template <bool SH, class T>
__device__ __forceinline__ T ld_page(const char* p) {
  if constexpr (SH) return *(global_ptr<T>)p;
  return __builtin_nontemporal_load((global_ptr<T>)p);
}

// ---------------------------------------------------------------------------------- few columns
// One token per sequence, or a few: every position's K and V comes once from memory and is used for
// at most 32 columns, so memory bounds it (INT8, head dim 128: 8.4 KB per pair of pages and kv head for 24 matrix
// instructions with 16 columns, 32 with 32, 48 with fp32 rows).  A workgroup takes a tile of 16 NT columns over a share of the span's
// pages; each of its 4 waves walks a run of pages by itself, straight from memory into operands (the
// page layout makes every load contiguous), two pages ahead of the pair that it computes; no barrier
// until the waves' (m, l, O) are joined in LDS.
// INT8, 8B heads, 64 sequences of 3,000-14,000 positions: 193 us, 5.9 TB/s (a copy reaches 5.07); 7B heads, one
// sequence of 14,336: 10.2-10.6 us with the join, mostly latency: a round of loads each for the arguments, the queries
// and the first pages, some 1 us per pair of pages, the join's launch.  Workgroups of 8 waves were slower
// at every size measured (12.1 and 208 us there), and so was a third pair in flight.
// SH: a span of the launch has several tiles.  They read the same pages, so these stay in the caches (without SH every
// load is non-temporal: 33 sequences of 3,000-14,000 positions, 16 rows, two tiles, 219 us; 195 so; 1,000 rows of an fp32
// pool behind 8,000 positions 125 and 92 us), and the tiles of a page share an XCD (8 rows of the 7B heads behind
// 14,001, bf16 pool, 18.7 and 15.8 us).  Where each page is read once, cached loads cost 7%: 32 sequences, 5 rows, 94
// us against 87.
// (bf16 pools and rows: 254 registers, so that two workgroups fit a CU; left to itself the compiler takes 257: 8 sequences of
// 3,000-14,000 50.8 and 52.2 us.)
template <class KT, class IT, int HD, int NT, bool SH>
__global__ __launch_bounds__(256, NT == 1 && sizeof(KT) == 2 && sizeof(IT) == 2 ? 2 : 1) void k_attend_rows(AttendArgs a) {
  constexpr int PARTS = std::is_same_v<IT, float> ? 3 : 1;    // of a query
  constexpr int WP = PARTS == 3 ? 3 : NT == 1 ? 2 : 1;        // of a weight
  constexpr int KP = std::is_same_v<KT, float> ? 3 : 1;       // of a key or value
  constexpr bool I8 = std::is_same_v<KT, i8_t>;
  constexpr bool INF = KP == 3 || (WP > 1 && sizeof(KT) == 2);  // infinities meet parts (8-bit pools have none)
  constexpr int NS = HD / 32, ND = HD / 16, NC = 16 * NT;
  constexpr int OS = HD + 4;  // LDS row stride (floats): 16 rows fall in different banks
  constexpr int ES = (int)sizeof(KT);
  __shared__ __align__(16) float s_o[4 * NC * OS];
  __shared__ float s_m[4 * NC], s_l[4 * NC];

  const unsigned item = blockIdx.x / (unsigned)a.hkv;
  const AttendSpan sp = item_span(a.n_spans, item);
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  const int lc = l & 15, lg = l >> 4;
  const int ncol = sp.n * a.G;
  int split = (int)(item - sp.first), kvh = (int)(blockIdx.x - item * a.hkv), tile = 0;
  if constexpr (SH) {  // the tiles that read the same pages are 8 workgroups apart, on one XCD and its L2
    const int tiles = (ncol + NC - 1) / NC, block = split * a.hkv + kvh, group = block / (8 * tiles);
    const int rest = block - group * 8 * tiles, across = min(8, sp.nsplit * a.hkv - 8 * group), nth = rest / across;
    const int pair = 8 * group + rest - nth * across;
    split = pair / a.hkv;
    kvh = pair - split * a.hkv;
    tile = tiles - 1 - nth;  // (the last tile has the most keys: first)
  }
  const int col0 = tile * NC;
  const int row_a = col0 / a.G, row_b = min(col0 + NC, ncol) - 1;  // first row, last column
  const int row_z = row_b / a.G;                                   // last row
  // the tile's keys, its pages and this wave's run of them
  const int klo = a.window > 0 ? max(sp.kb, sp.pos + row_a - a.window + 1) : sp.kb;
  const int khi = a.causal ? min(sp.ke, sp.pos + row_z + 1) : sp.ke;
  const int pg0 = klo >> 4, pg1 = khi > klo ? (khi + 15) >> 4 : pg0;
  const int share = (pg1 - pg0 + sp.nsplit - 1) / sp.nsplit;
  const int s0 = pg0 + split * share, s1 = min(s0 + share, pg1);
  const int run = (max(s1 - s0, 0) + 3) / 4;
  const int p0 = s0 + w * run, p1 = min(p0 + run, s1);
  const int* bt = a.bt + (size_t)sp.seq * a.max_pps;
  // pages that every column of the tile sees whole: [f0, f1)
  const int flo = a.window > 0 ? max(sp.kb, sp.pos + row_z - a.window + 1) : sp.kb;
  const int fhi = a.causal ? min(sp.ke, sp.pos + row_a + 1) : sp.ke;

  int cpos[NT], clo[NT];  // a column's last and first key (nothing seen: last before first)
  int crow[NT];
  bf16x8 q[NT][NS][PARTS];
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    const int c = min(col0 + 16 * u + lc, ncol - 1), r = c / a.G, h = kvh * a.G + c - r * a.G;
    crow[u] = r;
    cpos[u] = a.causal ? min(sp.ke - 1, sp.pos + r) : sp.ke - 1;
    clo[u] = a.window > 0 ? max(sp.kb, sp.pos + r - a.window + 1) : sp.kb;
    const int64_t e = (sp.row0 + r) * a.q_row + h * a.q_head + 8 * lg;
#pragma unroll
    for (int s = 0; s < NS; ++s) ld_query8<IT, PARTS>(a, e + 32 * s, q[u][s]);
  }
  float m[NT], ls[NT];
  f32x4 o[NT][ND];
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    m[u] = -INFINITY;
    ls[u] = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[u][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Raw words of a pair of pages: K (position lc, dims 32 s + 8 lg ..), V (dims 16 d + lc, positions 4 lg ..).
  using KRaw = std::conditional_t<ES == 1, u32x2, u32x4>;
  using VRaw = std::conditional_t<ES == 1, uint32_t, std::conditional_t<ES == 2, u32x2, u32x4>>;
  constexpr int KW = ES == 4 ? 2 : 1;
  struct Pair {
    KRaw k[2][NS][KW];
    VRaw v[2][ND];
    f32x4 ks[2], vs[2];
  };
  Pair buf[2];
  // The next pair's page ids, through the scalar unit.  Past the run they are its last page's again: a pair's
  // loads are always the same number, so that the wait for one pair leaves the next one's in flight (behind
  // a branch around them every wait is for all loads).
  int id[2] = {0, 0};
  auto look = [&](int pg) {
#pragma unroll
    for (int x = 0; x < 2; ++x) id[x] = ld_const<int>(bt + min(pg + x, p1 - 1));
  };
  auto load = [&](Pair& b, int pg) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int pid = __builtin_amdgcn_readfirstlane(id[x]);
      const size_t slot = ((size_t)a.layer * a.num_pages + pid) * a.hkv + kvh;
      const char* kb = (const char*)a.kpool + slot * (16 * HD * ES);
      const char* vb = (const char*)a.vpool + slot * (16 * HD * ES);
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int y = 0; y < KW; ++y)
          b.k[x][s][y] = ld_page<SH, KRaw>(kb + (s * 512 + 8 * l) * ES + 16 * y);
#pragma unroll
      for (int d = 0; d < ND; ++d) b.v[x][d] = ld_page<SH, VRaw>(vb + (d * 256 + 4 * l) * ES);
      if constexpr (I8) {
        b.ks[x] = ld_global<f32x4>((const char*)a.kpool + a.scales + slot * 64 + 16 * lg);
        b.vs[x] = ld_global<f32x4>((const char*)a.vpool + a.scales + slot * 64 + 16 * lg);
      }
    }
    look(pg + 2);
  };
  auto key = [&](const KRaw* raw, bf16x8* k, auto careful) {
    if constexpr (ES == 1) {
      uint32_t w4[4];
      if constexpr (I8) {
        i8x4_to_bf16x4(raw[0][0], w4[0], w4[1]);
        i8x4_to_bf16x4(raw[0][1], w4[2], w4[3]);
      } else {
        fp8x4_to_bf16x4(raw[0][0], w4[0], w4[1]);
        fp8x4_to_bf16x4(raw[0][1], w4[2], w4[3]);
      }
      k[0] = __builtin_bit_cast(bf16x8, u32x4{w4[0], w4[1], w4[2], w4[3]});
    } else if constexpr (ES == 2) {
      k[0] = __builtin_bit_cast(bf16x8, raw[0]);
    } else {
      u32x4 p[3];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t s[3];
        uint32_t a = raw[i >> 1][2 * (i & 1)], b = raw[i >> 1][2 * (i & 1) + 1];
        if constexpr (decltype(careful)::value) a = quiet(a), b = quiet(b);
        split3(__uint_as_float(a), __uint_as_float(b), s);
#pragma unroll
        for (int z = 0; z < 3; ++z) p[z][i] = s[z];
      }
#pragma unroll
      for (int z = 0; z < KP; ++z) k[z] = __builtin_bit_cast(bf16x8, p[z]);
    }
  };
  // dims 16 d + lc of positions 4 lg .. of both pages
  auto value = [&](const VRaw& va, const VRaw& vb, bf16x8* v, auto careful) {
    if constexpr (ES == 1) {
      uint32_t w4[4];
      if constexpr (I8) {
        i8x4_to_bf16x4(va, w4[0], w4[1]);
        i8x4_to_bf16x4(vb, w4[2], w4[3]);
      } else {
        fp8x4_to_bf16x4(va, w4[0], w4[1]);
        fp8x4_to_bf16x4(vb, w4[2], w4[3]);
      }
      v[0] = __builtin_bit_cast(bf16x8, u32x4{w4[0], w4[1], w4[2], w4[3]});
    } else if constexpr (ES == 2) {
      v[0] = __builtin_bit_cast(bf16x8, u32x4{va[0], va[1], vb[0], vb[1]});
    } else {
      u32x4 p[3];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t s[3];
        const VRaw& src = i < 2 ? va : vb;
        uint32_t a = src[2 * (i & 1)], b = src[2 * (i & 1) + 1];
        if constexpr (decltype(careful)::value) a = quiet(a), b = quiet(b);
        split3(__uint_as_float(a), __uint_as_float(b), s);
#pragma unroll
        for (int z = 0; z < 3; ++z) p[z][i] = s[z];
      }
#pragma unroll
      for (int z = 0; z < KP; ++z) v[z] = __builtin_bit_cast(bf16x8, p[z]);
    }
  };
  // products of parts i and j with i + j < 3 (the others are below 2^-24)
  auto mma = [&](const bf16x8* x, const auto& y, f32x4 acc, auto careful) {
#pragma unroll
    for (int i = KP - 1; i >= 0; --i)
#pragma unroll
      for (int j = (int)std::extent_v<std::remove_reference_t<decltype(y)>> - 1; j >= 0; --j) {
        if (i + j >= 3) continue;
        if constexpr (decltype(careful)::value)  // (only the leading parts meet an infinity)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(i + j > 0 ? finite_parts(x[i], x[0]) : x[0],
                                                        i + j > 0 ? finite_parts(y[j], y[0]) : y[0], acc, 0, 0, 0);
        else
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], y[j], acc, 0, 0, 0);
      }
    return acc;
  };
  auto compute = [&](const Pair& b, int pg, auto careful) {
    const bool whole = 16 * pg >= flo && 16 * pg + 32 <= fhi && pg + 1 < p1;  // (uniform)
    f32x4 s[NT][2];
#pragma unroll
    for (int u = 0; u < NT; ++u) s[u][0] = s[u][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        bf16x8 kk[KP];
        key(b.k[x][k], kk, careful);
#pragma unroll
        for (int u = 0; u < NT; ++u) s[u][x] = mma(kk, q[u][k], s[u][x], careful);
      }
    bf16x8 p[NT][WP];
    uint32_t seen[NT];  // this lane's 8 positions (bits 0-3 page pg, 4-7 page pg + 1)
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      float sv[8], mx = -INFINITY;
      seen[u] = 0xff;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) sv[4 * x + i] = s[u][x][i] * (I8 ? b.ks[x][i] * a.scale_log2 : a.scale_log2);
      if (!whole) {
        seen[u] = 0;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int t = 16 * (pg + x) + 4 * lg + i;
            const bool ok = t >= clo[u] && t <= cpos[u] && pg + x < p1;
            seen[u] |= (ok ? 1u : 0u) << (4 * x + i);
            sv[4 * x + i] = ok ? sv[4 * x + i] : -INFINITY;
          }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) mx = fmaxf(mx, sv[i]);
      mx = max_x32(max_x16(mx));
      const bool grow = mx > m[u];
      if (__ballot(grow)) {
        const float mn = grow ? mx + kSlack : m[u];
        const float alpha = grow ? __builtin_amdgcn_exp2f(m[u] - mn) : 1.f;  // (m = -inf: 0)
        ls[u] *= alpha;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[u][d] *= alpha;
        m[u] = mn;
      }
      const float mu = m[u] == -INFINITY ? 0.f : m[u];
      float pv[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = __builtin_amdgcn_exp2f(sv[i] - mu);
        ls[u] += e;
        pv[i] = e;
        if constexpr (I8) pv[i] = whole || ((seen[u] >> i) & 1) ? e * b.vs[i >> 2][i & 3] : 0.f;
      }
      u32x4 pw[WP];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (WP < 3) {
          const uint32_t t = pw[0][i] = pk_bf16(pv[2 * i], pv[2 * i + 1]);
          if constexpr (WP == 2) pw[1][i] = pk_bf16(pv[2 * i] - __uint_as_float(t << 16), pv[2 * i + 1] - __uint_as_float(t & 0xffff0000u));
        } else {
          uint32_t s3[3];
          split3(pv[2 * i], pv[2 * i + 1], s3);
#pragma unroll
          for (int k = 0; k < WP; ++k) pw[k][i] = s3[k];
        }
      }
#pragma unroll
      for (int k = 0; k < WP; ++k) p[u][k] = __builtin_bit_cast(bf16x8, pw[k]);
    }
    bool odd = false;
    if (!I8 && (decltype(careful)::value || !whole)) {  // an infinite or NaN V anywhere in the pair?
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          if constexpr (ES == 1) {
            uint32_t lo, hi;
            fp8x4_to_bf16x4(b.v[x][d], lo, hi);
            odd |= odd_bf16(lo) || odd_bf16(hi);
          } else if constexpr (ES == 2) {
            odd |= odd_bf16(b.v[x][d][0]) || odd_bf16(b.v[x][d][1]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) odd |= (b.v[x][d][i] & 0x7f800000u) == 0x7f800000u;
          }
        }
    }
    if (!__ballot(odd)) {
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        bf16x8 v[KP];
        value(b.v[0][d], b.v[1][d], v, careful);
#pragma unroll
        for (int u = 0; u < NT; ++u) o[u][d] = mma(v, p[u], o[u][d], careful);
      }
    } else if constexpr (!I8) {
      // row by row: V of the positions that the row does not see is zero, and the row's columns take
      // the result (a column's sums depend on its own weights only)
      for (int r = row_a; r <= row_z; ++r) {
        const int last = min(a.causal ? min(sp.ke - 1, sp.pos + r) : sp.ke - 1, 16 * p1 - 1);
        const int begin = a.window > 0 ? max(sp.kb, sp.pos + r - a.window + 1) : sp.kb;
        uint32_t vis = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = 16 * (pg + (i >> 2)) + 4 * lg + (i & 3);
          vis |= (t >= begin && t <= last ? 1u : 0u) << i;
        }
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          VRaw va = b.v[0][d], vb = b.v[1][d];
          if constexpr (ES == 1) {
            uint32_t ma = 0, mb = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              ma |= (vis >> i) & 1 ? 0xffu << (8 * i) : 0u;
              mb |= (vis >> (4 + i)) & 1 ? 0xffu << (8 * i) : 0u;
            }
            va &= ma;
            vb &= mb;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t keep = ES == 2 ? 0xffffu << (16 * (i & 1)) : 0xffffffffu;
              if (!((vis >> i) & 1)) va[ES == 2 ? i >> 1 : i] &= ~keep;
              if (!((vis >> (4 + i)) & 1)) vb[ES == 2 ? i >> 1 : i] &= ~keep;
            }
          }
          bf16x8 v[KP];
          value(va, vb, v, careful);
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            const f32x4 t = mma(v, p[u], o[u][d], careful);
            if (crow[u] == r) o[u][d] = t;
          }
        }
      }
    }
  };
  if (p0 < p1) {
    look(p0);
    load(buf[0], p0);
    for (int pg = p0; pg < p1; pg += 4) {
      load(buf[1], pg + 2);
      compute(buf[0], pg, std::false_type{});
      if (pg + 2 >= p1) break;
      load(buf[0], pg + 4);
      compute(buf[1], pg + 2, std::false_type{});
    }
    if constexpr (INF) {  // a sum that is infinite or NaN stays so: the run once more, parts and infinities apart
      float z = 0.f;
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        z = fmaf(ls[u], 0.f, z);
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) z = fmaf(o[u][d][i], 0.f, z);
      }
      if (__builtin_expect(__ballot(z != 0.f) != 0, 0)) {
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          m[u] = -INFINITY;
          ls[u] = 0.f;
#pragma unroll
          for (int d = 0; d < ND; ++d) o[u][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll 1
        for (int pg = p0; pg < p1; pg += 2) {
          look(pg);
          load(buf[0], pg);
          compute(buf[0], pg, std::true_type{});
        }
      }
    }
  }

  // ---- the waves' (m, l, O) joined, in wave order
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    const float lsum = sum_x32(sum_x16(ls[u]));
    const int c = w * NC + 16 * u + lc;
#pragma unroll
    for (int d = 0; d < ND; ++d) *(f32x4*)(s_o + c * OS + 16 * d + 4 * lg) = o[u][d];
    if (lg == 0) {
      s_m[c] = m[u];
      s_l[c] = lsum;
    }
  }
  __syncthreads();
  constexpr int CH = HD / 4;
  const int cols = min(NC, ncol - col0);
  for (int i = tid; i < cols * CH; i += 256) {
    const int c = i / CH, d4 = i % CH;
    float M = -INFINITY;
#pragma unroll
    for (int v = 0; v < 4; ++v) M = fmaxf(M, s_m[v * NC + c]);
    float L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float mv = s_m[v * NC + c];
      const float f = mv == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mv - M);
      L += s_l[v * NC + c] * f;
      acc += *(const f32x4*)(s_o + (v * NC + c) * OS + 4 * d4) * f;
    }
    const int r = (col0 + c) / a.G, h = kvh * a.G + col0 + c - r * a.G;
    if (sp.nsplit == 1) {
      st_out4<IT>(a, sp.row0 + r, h, 4 * d4, normed(acc, L));
      if (d4 == 0 && a.lse != nullptr)
        a.lse[(size_t)(sp.row0 + r) * a.hq + h] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
    } else {
      const size_t part = sp.part0 + ((size_t)r * a.hq + h) * sp.nsplit + split;
      *(f32x4*)(a.part + part * HD + 4 * d4) = acc;
      if (d4 == 0) *(float2*)(a.ml + part * 2) = make_float2(M, L);
    }
  }
}

// ---------------------------------------------------------------------------------- many columns
// Chunks of many rows: the matrix cores' work.  A workgroup of 8 waves takes a tile of 256 columns, 32 to a
// wave, over a share of the tile's pages, 4 pages (64 positions) at a time: the waves fetch them together
// (half of them K, half V; the next 4 pages' words are in flight while these are computed), convert them
// to bf16 once for all 256 columns and leave them in one of two LDS buffers in operand order; one
// barrier per 4 pages.  v_mfma_f32_32x32x16_bf16: a wave's S^T is 2 x (32 positions x 32 columns), and a page's
// 16 positions are one contraction step of the second product.
// Bound by matrix and vector instructions together, which a SIMD overlaps only in part (32 rows x 64
// positions: 32 matrix instructions of 32 cycles, some 270 vector ones).  4,096 rows of 32 heads behind
// 12,288 positions, INT8: 1.00-1.14 ms from card to card, 840-960 TFLOP/s, where a large bf16 matrix product reaches
// 1,200-1,370; 1.73 ms with the row kernel.  What it took: accumulators that no rare branch copies (1.28 -> 1.07 ms),
// operands read six products ahead (4%), integer V scales inside the exponent (3%).
// fp32 rows: 3 parts of each query and weight, the same 32 columns.
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <class KT, class IT, int HD>
__global__ __launch_bounds__(512) void k_attend_tile(AttendArgs a) {
  constexpr int PARTS = std::is_same_v<IT, float> ? 3 : 1;
  constexpr bool I8 = std::is_same_v<KT, i8_t>;
  constexpr bool INF = PARTS == 3 && sizeof(KT) == 2;  // infinities meet parts
  constexpr int ES = (int)sizeof(KT), NK = HD / 16, ND = HD / 32, SP = 4;  // SP: pages of a step
  constexpr int PB = 32 * HD;             // bytes of a page's K or V in LDS (bf16)
  constexpr int NL = 16 * HD * ES / 1024; // 16-byte loads per lane for a page's K or V
  static_assert(ES <= 2, "fp32 pools: the row kernel");
  constexpr int KB = PB + 128;            // (of a K page: two pages are read at once, from different banks)
  __shared__ __align__(16) char s_k[2][SP * KB], s_v[2][SP * PB];
  __shared__ __align__(16) float s_ks[2][16 * SP], s_vs[2][16 * SP], s_lv[2][16 * SP];
  __shared__ __align__(16) int s_odd[2][SP];

  const unsigned item = blockIdx.x / (unsigned)a.hkv;
  const int kvh = (int)(blockIdx.x - item * a.hkv);
  const AttendSpan sp = item_span(a.n_spans, item);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int lc = l & 31, h = l >> 5;
  const int ncol = sp.n * a.G, tiles = (ncol + kAttendTileCols - 1) / kAttendTileCols;
  const int local = (int)(item - sp.first), split = local % sp.nsplit;
  const int tile = tiles - 1 - local / sp.nsplit;  // (the last tile has the most keys: first)
  const int col0 = tile * kAttendTileCols;
  auto first_key = [&](int row) { return a.window > 0 ? max(sp.kb, sp.pos + row - a.window + 1) : sp.kb; };
  auto end_key = [&](int row) { return a.causal ? min(sp.ke, sp.pos + row + 1) : sp.ke; };
  const int klo = first_key(col0 / a.G), khi = end_key((min(col0 + kAttendTileCols, ncol) - 1) / a.G);
  const int pg0 = klo >> 4, pg1 = khi > klo ? (khi + 15) >> 4 : pg0;
  const int share = ((pg1 - pg0 + sp.nsplit - 1) / sp.nsplit + SP - 1) / SP * SP;
  const int s0 = pg0 + split * share, s1 = min(s0 + share, pg1);
  const int* bt = a.bt + (size_t)sp.seq * a.max_pps;

  // this wave's columns
  const int wc0 = col0 + 32 * w, wcz = min(wc0 + 32, ncol) - 1;
  const int row_a = min(wc0, ncol - 1) / a.G, row_z = max(wcz, 0) / a.G;
  const int flo = first_key(row_z), fhi = min(end_key(row_a), 16 * s1);  // keys that all of them see
  const int c = min(wc0 + lc, ncol - 1), row = c / a.G, head = kvh * a.G + c - row * a.G;
  const int clo = first_key(row), chi = min(end_key(row), 16 * s1);
  bf16x8 q[NK][PARTS];
  {
    const int64_t e = (sp.row0 + row) * a.q_row + head * a.q_head + 8 * h;
#pragma unroll
    for (int k = 0; k < NK; ++k) ld_query8<IT, PARTS>(a, e + 16 * k, q[k], a.scale_log2 < 0.f ? 0x80000000u : 0u);
  }
  float m = -INFINITY, ls = 0.f;
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  // the scale, positive (the queries carry its sign).  Zero is taken as the smallest number above it: a score of
  // -infinity stays one, and the largest finite one comes to 2^-21.
  const float sc = fmaxf(fabsf(a.scale_log2), 0x1p-149f);

  // staging: waves 0-3 K, 4-7 V of page w % 4 of the step
  const bool st_v = w >= SP;
  const int st_p = w & (SP - 1);
  u32x4 raw[NL];
  float raw_s = 0.f;
  auto fetch = [&](int pg) {
    const int pid = ld_const<int>(bt + min(pg + st_p, s1 - 1));  // (past the share: its last page again, unseen)
    const size_t slot = ((size_t)a.layer * a.num_pages + pid) * a.hkv + kvh;
    const char* pool = (const char*)(st_v ? a.vpool : a.kpool);
    const char* b = pool + slot * (16 * HD * ES) + 16 * l;
#pragma unroll
    for (int i = 0; i < NL; ++i) raw[i] = ld_global<u32x4>(b + 1024 * i);
    if constexpr (I8) raw_s = ld_global<float>(pool + a.scales + slot * 64 + 4 * (l & 15));
  };
  auto convert = [&](uint32_t x, uint32_t& lo, uint32_t& hi) {
    if constexpr (I8)
      i8x4_to_bf16x4(x, lo, hi);
    else
      fp8x4_to_bf16x4(x, lo, hi);
  };
  // What V holds past the last key is taken as zero.  A page with an odd value is flagged; unless it is
  // asked for as it is, its V is zero too, and its step is left for the end.  Odd are infinities and NaN,
  // and V scales s of an integer page outside 2^-36 .. 2^36: there the weights p s are computed as
  // exp2(score + log2 s), and the sum of the p as that of the p s times 1 / s, which saves an operation per
  // weight but would lose some p below 2^-46 of the largest (126 - 8 of m - 2 x 36) if the scales lay further apart.  (All zeros:
  // any scale will do.)
  auto stage = [&](int buf, int pg, bool as_is) {
    if (!st_v) {  // as in the page: chunk (8 dims, position) at 16 bytes each
      char* d = s_k[buf] + st_p * KB;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        if constexpr (ES == 2) {
          *(u32x4*)(d + (64 * i + l) * 16) = raw[i];
        } else {
          uint32_t t[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) convert(raw[i][e], t[2 * e], t[2 * e + 1]);
          *(u32x4*)(d + (64 * i + l) * 32) = u32x4{t[0], t[1], t[2], t[3]};
          *(u32x4*)(d + (64 * i + l) * 32 + 16) = u32x4{t[4], t[5], t[6], t[7]};
        }
      }
      if (I8 && l < 16) s_ks[buf][16 * st_p + l] = raw_s * sc;
    } else {  // positions 4 x .. 4 x + 3 of a dim go to half x / 2 of its 16 bytes in plane x % 2
      char* d = s_v[buf] + st_p * PB;
      const int left = sp.ke - 16 * (pg + st_p);  // keys of the page
      if (__builtin_expect(left < 16, 0)) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int n = min(max(left - 4 * ((64 * i + l) / (ES == 2 ? 8 : 4) % 4), 0), 4);  // keys of the 4
          const uint64_t keep = n == 4 ? ~0ull : (1ull << (8 * ES * n)) - 1;
          raw[i] &= ES == 2 ? u32x4{(uint32_t)keep, (uint32_t)(keep >> 32), (uint32_t)keep, (uint32_t)(keep >> 32)}
                            : u32x4{(uint32_t)keep, (uint32_t)keep, (uint32_t)keep, (uint32_t)keep};
        }
        if ((l & 15) >= left) raw_s = 0.f;
      }
      bool odd = I8 && raw_s != 0.f && !(raw_s >= 0x1p-36f && raw_s <= 0x1p36f);
      if constexpr (!I8)
#pragma unroll
        for (int i = 0; i < NL; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (ES == 2) {
              odd |= odd_bf16(raw[i][e]);
            } else {  // E4M3: a NaN is all ones below the sign
              const uint32_t x = raw[i][e] & 0x7f7f7f7fu;
              odd |= ((x + 0x01010101u) & 0x80808080u) != 0;
            }
          }
      const bool any = __ballot(odd) != 0;
      if (l == 0) s_odd[buf][st_p] = any;
      if (__builtin_expect(any && !as_is, 0)) {
#pragma unroll
        for (int i = 0; i < NL; ++i) raw[i] = u32x4{0, 0, 0, 0};
        raw_s = 0.f;
      }
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int k = 64 * i + l;
        if constexpr (ES == 2) {
          const int d0 = k / 32 * 16 + 2 * (k % 8), x = k / 8 % 4;
          char* b = d + ((x & 1) * HD + d0) * 16 + (x >> 1) * 8;
          *(u32x2*)b = u32x2{raw[i][0], raw[i][1]};
          *(u32x2*)(b + 16) = u32x2{raw[i][2], raw[i][3]};
        } else {
          const int d0 = k / 16 * 16 + 4 * (k % 4), x = k / 4 % 4;
          char* b = d + ((x & 1) * HD + d0) * 16 + (x >> 1) * 8;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t lo, hi;
            convert(raw[i][e], lo, hi);
            *(u32x2*)(b + 16 * e) = u32x2{lo, hi};
          }
        }
      }
      if (I8 && l < 16) {
        const float s = raw_s == 0.f ? 0x1p-36f : raw_s;
        s_lv[buf][16 * st_p + l] = __builtin_amdgcn_logf(s);
        s_vs[buf][16 * st_p + l] = as_is ? raw_s : 1.f / s;
      }
    }
  };
  auto is_odd = [&](int buf) {  // (every wave sees the same)
    const u32x4 f = *(const u32x4*)s_odd[buf];
    return __builtin_amdgcn_readfirstlane(f[0] | f[1] | f[2] | f[3]) != 0;
  };
  // Scores of a step (64 positions from 16 pg): lane (column lc, half h), element i of s[x] is position
  // 32 x + 8 (i / 4) + 4 h + i % 4.  Integer pages: in exp2 units, plus log2 of the position's V scale (as it
  // is: without); otherwise before the scale.
  f32x16 s[2];
  auto scores = [&](int buf, bool as_is, auto careful) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[x][i] = 0.f;
      const char* b = s_k[buf] + (2 * x + (lc >> 4)) * KB + (lc & 15) * 16 + h * 256;
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        const bf16x8 kk = *(const bf16x8*)(b + 512 * k);
#pragma unroll
        for (int z = PARTS - 1; z >= 0; --z)
          s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decltype(careful)::value && z > 0 ? finite_parts(kk, kk) : kk, q[k][z], s[x], 0, 0, 0);
      }
    }
    if constexpr (I8)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const f32x4 ks = *(const f32x4*)(s_ks[buf] + 32 * x + 8 * b + 4 * h);
          const f32x4 lv = as_is ? f32x4{0.f, 0.f, 0.f, 0.f} : *(const f32x4*)(s_lv[buf] + 32 * x + 8 * b + 4 * h);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[x][4 * b + i] = fmaf(s[x][4 * b + i], ks[i], lv[i]);
        }
  };
  // -infinity for positions outside lo .. hi-1
  auto hide = [&](int pg, int lo, int hi) {
    lo -= 16 * pg + 4 * h;
    hi -= 16 * pg + 4 * h;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int t = 32 * x + 8 * (i >> 2) + (i & 3);
        if (t < lo || t >= hi) s[x][i] = -INFINITY;
      }
  };
  auto raise_max = [&]() {
    float mx = -INFINITY;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[x][i]);
    mx = max_x32(mx) * (I8 ? 1.f : sc);
    const bool grow = mx > m;
    if (__builtin_expect(__ballot(grow) != 0, 0)) {
      const float mn = grow ? mx + kSlack : m;
      const float alpha = grow ? __builtin_amdgcn_exp2f(m - mn) : 1.f;
      ls *= alpha;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= alpha;
      m = mn;
    }
  };
  u32x4 pw[2][PARTS];
  auto weights = [&](int buf, int y, bool as_is) {  // of page y of the step: elements 8 (y % 2) .. of s[y / 2]
    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      float pv[4];
      f32x4 vs = {1.f, 1.f, 1.f, 1.f};
      if constexpr (I8) vs = *(const f32x4*)(s_vs[buf] + 16 * y + 8 * b + 4 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = s[y >> 1][8 * (y & 1) + 4 * b + i];
        const float e = __builtin_amdgcn_exp2f(I8 ? x - mu : fmaf(x, sc, -mu));
        ls = I8 && !as_is ? fmaf(e, vs[i], ls) : ls + e;
        pv[i] = I8 && as_is ? e * vs[i] : e;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (PARTS == 1) {
          pw[y & 1][0][2 * b + i] = pk_bf16(pv[2 * i], pv[2 * i + 1]);
        } else {
          uint32_t s3[3];
          split3(pv[2 * i], pv[2 * i + 1], s3);
#pragma unroll
          for (int z = 0; z < PARTS; ++z) pw[y & 1][z][2 * b + i] = s3[z];
        }
      }
    }
  };
  auto product = [&](u32x4 vw, int y, f32x16 acc, auto careful) {
    const bf16x8 v = __builtin_bit_cast(bf16x8, vw);
#pragma unroll
    for (int z = PARTS - 1; z >= 0; --z)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decltype(careful)::value && z > 0 ? finite_parts(v, v) : v,
                                                    __builtin_bit_cast(bf16x8, pw[y & 1][z]), acc, 0, 0, 0);
    return acc;
  };
  using Careful = std::bool_constant<INF>;
  // What is rare (positions that not every column sees, a maximum that moves) stands in branches of its own
  // that change the registers in place, and odd steps come after all others: so the loop keeps its
  // accumulators where they are.
  auto step = [&](int buf, int pg, bool odd) {
    scores(buf, false, std::false_type{});
    if constexpr (PARTS == 1) {  // operands ahead of their products
      __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
      for (int i = 0; i < 2 * NK; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    if (__builtin_expect(odd || 16 * pg < flo || 16 * (pg + SP) > fhi, 0)) hide(pg, clo, odd ? 0 : chi);
    raise_max();
    const char* vb = s_v[buf] + (h * HD + lc) * 16;
    weights(buf, 0, false);
#pragma unroll
    for (int y = 0; y < SP; ++y) {
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] = product(*(const u32x4*)(vb + y * PB + d * 512), y, o[d], std::false_type{});
      if (y + 1 < SP) weights(buf, y + 1, false);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // A step with odd values, row by row as in the row kernel: V of the positions that the row does not see is
  // zero (an integer page: their weights), and the row's columns take the result; parts and infinities apart.  (INF, V
  // not odd: all columns at once.)
  auto odd_step = [&](int buf, int pg, bool odd) {
    if constexpr (!INF) odd = true;
    scores(buf, true, Careful{});
    hide(pg, clo, chi);
    raise_max();
    const char* vb = s_v[buf] + (h * HD + lc) * 16;
#pragma unroll
    for (int y = 0; y < SP; ++y) {
      weights(buf, y, true);
#pragma unroll 1
      for (int r = odd ? row_a : row_z; r <= row_z; ++r) {
        const int begin = first_key(r), end = min(end_key(r), 16 * s1);
        u32x4 keep;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int t = 16 * (pg + y) + 8 * (j >> 2) + 4 * h + (j & 3);
          const uint32_t k16 = !odd || (t >= begin && t < end) ? 0xffffu : 0u;
          keep[j >> 1] = (j & 1) ? keep[j >> 1] | (k16 << 16) : k16;
        }
        if constexpr (I8)  // (a lane's own column decides; the others' results are not taken)
#pragma unroll
          for (int z = 0; z < PARTS; ++z)
            if (row == r) pw[y & 1][z] &= keep;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const u32x4 v = *(const u32x4*)(vb + y * PB + d * 512);
          const f32x16 t = product(I8 ? v : v & keep, y, o[d], Careful{});
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] = row == r || !odd ? t[i] : o[d][i];
        }
      }
    }
  };
  if (s0 < s1) {  // (workgroup-uniform)
    fetch(s0);
    stage(0, s0, false);
    __syncthreads();
    int buf = 0;
    bool left = false;
    for (int pg = s0; pg < s1; pg += SP, buf ^= 1) {
      const bool more = pg + SP < s1, odd = is_odd(buf);
      left |= odd;
      if (more) fetch(pg + SP);
      step(buf, pg, odd);
      if (more) stage(buf ^ 1, pg + SP, false);
      __syncthreads();
    }
    bool again = false;
    if constexpr (INF) {  // a score is NaN, perhaps by its parts: all steps once more
      again = __syncthreads_or(ls != ls);
      if (__builtin_expect(again, 0)) {
        m = -INFINITY;
        ls = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
      }
    }
    if (__builtin_expect(left || again, 0)) {
#pragma unroll 1
      for (int pg = s0; pg < s1; pg += SP) {
        fetch(pg);
        stage(0, pg, true);
        __syncthreads();
        const bool odd = is_odd(0);
        if (odd || again) odd_step(0, pg, odd);
        __syncthreads();
      }
    }
  }
  if (wc0 + lc >= ncol) return;
  ls = sum_x32(ls);
  if (sp.nsplit == 1) {
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        st_out4<IT>(a, sp.row0 + row, head, 32 * d + 8 * b + 4 * h,
                    normed(f32x4{o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]}, ls));
    if (h == 0 && a.lse != nullptr)
      a.lse[(size_t)(sp.row0 + row) * a.hq + head] = ls == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(ls)) * kLn2;
  } else {
    const size_t part = sp.part0 + ((size_t)row * a.hq + head) * sp.nsplit + split;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *(f32x4*)(a.part + part * HD + 32 * d + 8 * b + 4 * h) =
            f32x4{o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
    if (h == 0) *(float2*)(a.ml + part * 2) = make_float2(m, ls);
  }
}

// ---------------------------------------------------------------------------------- the splits joined
// o = sum_s O_s 2^(m_s - M) / sum_s l_s 2^(m_s - M).  A workgroup per (row, head): HD / 4 lanes read a
// split's O with 16-byte loads, so that the workgroup's 4 waves take 8 (16 at head dim 64) splits at once,
// up to kAttendMaxSplits with all loads in flight together.
template <class IT, int HD>
__global__ __launch_bounds__(256) void k_attend_merge(AttendArgs a) {
  constexpr int LPS = HD / 4, SPP = 256 / LPS, PER = kAttendMaxSplits / SPP;
  __shared__ __align__(16) float s_o[4][HD];
  __shared__ float s_m[4], s_l[4];
  const unsigned item = blockIdx.x;
  const AttendSpan sp = item_span(a.n_spans, item);
  const unsigned local = item - sp.first;
  const int r = (int)(local / (unsigned)a.hq), h = (int)(local - (unsigned)r * a.hq);
  const size_t part = sp.part0 + (size_t)local * sp.nsplit;
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, d4 = tid % LPS, sl = tid / LPS;
  float mv[PER], lv[PER];
  f32x4 ov[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int s = i * SPP + sl;
    mv[i] = -INFINITY;
    lv[i] = 0.f;
    ov[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (s < sp.nsplit) {
      const float2 x = *(const float2*)(a.ml + (part + s) * 2);
      mv[i] = x.x;
      lv[i] = x.y;
      ov[i] = ld_global<f32x4>(a.part + (part + s) * HD + 4 * d4);
    }
  }
  float M = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) M = fmaxf(M, mv[i]);
  M = max_x32(LPS == 16 ? max_x16(M) : M);
  float L = 0.f;
  f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const float f = mv[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mv[i] - M);
    L += lv[i] * f;
    O += ov[i] * f;
  }
  if constexpr (LPS == 16) {
    L = sum_x16(L);
#pragma unroll
    for (int i = 0; i < 4; ++i) O[i] = sum_x16(O[i]);
  }
  L = sum_x32(L);
#pragma unroll
  for (int i = 0; i < 4; ++i) O[i] = sum_x32(O[i]);
  if (l < LPS) *(f32x4*)&s_o[w][4 * d4] = O;
  if (l == 0) {
    s_m[w] = M;
    s_l[w] = L;
  }
  __syncthreads();
  if (tid >= LPS) return;
  float Mt = -INFINITY, Lt = 0.f;
#pragma unroll
  for (int v = 0; v < 4; ++v) Mt = fmaxf(Mt, s_m[v]);
  f32x4 Ot = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const float f = s_m[v] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[v] - Mt);
    Lt += s_l[v] * f;
    Ot += *(const f32x4*)&s_o[v][4 * d4] * f;
  }
  st_out4<IT>(a, sp.row0 + r, h, 4 * d4, normed(Ot, Lt));
  if (d4 == 0 && a.lse != nullptr)
    a.lse[(size_t)(sp.row0 + r) * a.hq + h] = Lt == 0.f ? -INFINITY : (Mt + __builtin_amdgcn_logf(Lt)) * kLn2;
}

// The same for spans of at most kAttendFewSplits splits (chunks: many rows, few splits): HD / 4 lanes per (row, head)
// hold all of them; bounded by the partials' bytes.
template <class IT, int HD>
__global__ __launch_bounds__(256) void k_attend_merge_few(AttendArgs a) {
  constexpr int LPS = HD / 4, NG = 256 / LPS;
  const AttendSpan sp = item_span(a.n_spans, blockIdx.x);
  const unsigned local = (blockIdx.x - sp.first) * NG + threadIdx.x / LPS;
  if (local >= (unsigned)sp.n * a.hq) return;
  const int r = (int)(local / (unsigned)a.hq), h = (int)(local - (unsigned)r * a.hq), d4 = threadIdx.x % LPS;
  const size_t part = sp.part0 + (size_t)local * sp.nsplit;
  float mv[kAttendFewSplits], lv[kAttendFewSplits], M = -INFINITY, L = 0.f;
  f32x4 ov[kAttendFewSplits], O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < kAttendFewSplits; ++s) {
    const size_t at = part + min(s, sp.nsplit - 1);
    const float2 x = *(const float2*)(a.ml + at * 2);
    mv[s] = x.x;
    lv[s] = x.y;
    ov[s] = ld_global<f32x4>(a.part + at * HD + 4 * d4);
  }
#pragma unroll
  for (int s = 0; s < kAttendFewSplits; ++s) M = fmaxf(M, mv[s]);  // (the last one several times: the same maximum)
#pragma unroll
  for (int s = 0; s < kAttendFewSplits; ++s) {
    if (s >= sp.nsplit) break;
    const float f = mv[s] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mv[s] - M);
    L += lv[s] * f;
    O += ov[s] * f;
  }
  st_out4<IT>(a, sp.row0 + r, h, 4 * d4, normed(O, L));
  if (d4 == 0 && a.lse != nullptr)
    a.lse[(size_t)(sp.row0 + r) * a.hq + h] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
}

template <class KT, class IT, int HD>
static hipError_t launch_kind(int kind, const AttendArgs& a, hipStream_t s) {
  const dim3 grid(a.n_items * (unsigned)a.hkv), block(256);
  if (kind == 2) {
    if constexpr (sizeof(KT) <= 2) return launch_k(k_attend_tile<KT, IT, HD>, grid, dim3(512), s, a);
    return hipErrorInvalidValue;
  }
  if (kind == 1) {
    if constexpr (sizeof(KT) <= 2 && sizeof(IT) == 2)
      return a.shared ? launch_k(k_attend_rows<KT, IT, HD, 2, true>, grid, block, s, a)
                      : launch_k(k_attend_rows<KT, IT, HD, 2, false>, grid, block, s, a);
    return hipErrorInvalidValue;
  }
  return a.shared ? launch_k(k_attend_rows<KT, IT, HD, 1, true>, grid, block, s, a)
                  : launch_k(k_attend_rows<KT, IT, HD, 1, false>, grid, block, s, a);
}

hipError_t launch_attend(int kind, int kv_type, int io, int hd, const AttendArgs& a, hipStream_t s) {
  if (a.n_spans < 1 || a.n_spans > kAttendSpans || a.n_items < 1 || (hd != 64 && hd != 128)) return hipErrorInvalidValue;
  auto go = [&](auto kt) {
    using KT = decltype(kt);
    if (io == 1) return hd == 128 ? launch_kind<KT, bf16_t, 128>(kind, a, s) : launch_kind<KT, bf16_t, 64>(kind, a, s);
    return hd == 128 ? launch_kind<KT, float, 128>(kind, a, s) : launch_kind<KT, float, 64>(kind, a, s);
  };
  switch (kv_type) {
    case 0: return go(float{});
    case 1: return go(bf16_t{});
    case 2: return go(fp8_t{});
    default: return go(i8_t{});
  }
}

hipError_t launch_attend_merge(int io, int hd, bool few, const AttendArgs& a, hipStream_t s) {
  if (a.n_spans < 1 || a.n_spans > kAttendSpans || a.n_items < 1 || (hd != 64 && hd != 128)) return hipErrorInvalidValue;
  const dim3 grid(a.n_items), block(256);
  auto go = [&](auto it) {
    using IT = decltype(it);
    if (few)
      return hd == 128 ? launch_k(k_attend_merge_few<IT, 128>, grid, block, s, a) : launch_k(k_attend_merge_few<IT, 64>, grid, block, s, a);
    return hd == 128 ? launch_k(k_attend_merge<IT, 128>, grid, block, s, a) : launch_k(k_attend_merge<IT, 64>, grid, block, s, a);
  };
  return io == 1 ? go(bf16_t{}) : go(float{});
}

}  // namespace laser
