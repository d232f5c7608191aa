// Attention of a caller's query rows over the paged KV cache (laser_attend).
//
// Row i of a span sits at position pos + i and sees the keys t in [kb, ke) with t <= pos + i (causal)
// and t > pos + i - window (window > 0):
//   s_t = scale q.k_t,  m = max s_t,  l = sum exp(s_t - m),  o = sum exp(s_t - m) v_t / l,
//   lse = m + log l;  nothing seen: o = 0, lse = -inf.
// The keys are taken once, in exp2 units, with a running m and l per row.  m is only moved, and what
// has been summed rescaled, when a score exceeds it by more than kSlack: exp2 of up to that much keeps
// every sum far inside fp32, and the weights' relative rounding does not change.
//
// The G query heads of a kv head and the rows of a span are the columns of one matrix: column c is row
// c / G, head kvh G + c % G, so that K and V are read once for all of them.  Matrix-core products, K or V
// as the A operand:
//   S^T[t][c] = K[t][:] . Q[c][:],   O^T[d][c] += V^T[d][t] P^T[t][c];
// the second takes P^T as the first leaves it in its accumulators: which position stands in which slot
// of the contraction is free, as long as V is read in the same order.
// Types: K and V as bf16 (bf16, E4M3 and 8-bit integers are exact in it; an integer row's scale goes
// onto the scores, and onto the weights).  bf16 queries are exact; the weights are rounded to bf16, a
// relative 2^-9 each beside the 2^-9 of the bf16 output.  With fp32 queries and output, queries and weights
// (and fp32 K and V) are split into three bf16 parts, which hold all 24 bits.  m, l, O: fp32.
// A key that a row does not see may hold anything: its score is replaced, an integer row's weight too
// (whatever the scale), and where the stored V itself can be infinite or NaN, pages that not every
// column sees whole are looked through and, if one has such a value, taken row by row with the
// unseen positions' V zeroed.
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

// The span of a work item (spans are listed by their first item).
__device__ __forceinline__ int find_span(const AttendArgs& a, unsigned item) {
  const int lane = threadIdx.x & 63;
  const unsigned first = lane < a.n_spans ? a.sp[lane].first : 0xffffffffu;
  return __builtin_popcountll(__ballot(first <= item)) - 1;
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
template <class IT, int PARTS>
__device__ __forceinline__ void ld_query8(const AttendArgs& a, int64_t e, bf16x8* out) {
  if constexpr (std::is_same_v<IT, bf16_t>) {
    const uint16_t* p = (const uint16_t*)a.q + e;
    u32x4 w;
    if (a.q_vec) {
      w = ld_global<u32x4>(p);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
    }
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
      split3(x[i >> 1][2 * (i & 1)], x[i >> 1][2 * (i & 1) + 1], s);
#pragma unroll
      for (int k = 0; k < 3; ++k) w[k][i] = s[k];
    }
#pragma unroll
    for (int k = 0; k < PARTS; ++k) out[k] = __builtin_bit_cast(bf16x8, w[k]);
  }
}

__device__ __forceinline__ bool odd_bf16(uint32_t w) {  // one of a pair is infinite or NaN
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

}  // namespace

// ---------------------------------------------------------------------------------- few columns
// One token per sequence, or a few: every position's K and V comes once from memory and is used for
// at most 32 columns, so memory bounds it (8-bit keys at 14k positions: 8.4 KB per page and kv head
// for 64 matrix instructions).  A workgroup takes a tile of 16 NT columns over a share of the span's
// pages; each of its 4 waves walks a run of pages by itself, straight from memory into operands (the
// page layout makes every load contiguous), two pages ahead of the pair that it computes; no barrier
// until the waves' (m, l, O) are joined in LDS.
template <class KT, class IT, int HD, int NT>
__global__ __launch_bounds__(256) void k_attend_rows(AttendArgs a) {
  constexpr int PARTS = std::is_same_v<IT, float> ? 3 : 1;    // of a query or weight
  constexpr int KP = std::is_same_v<KT, float> ? 3 : 1;       // of a key or value
  constexpr bool I8 = std::is_same_v<KT, i8_t>;
  constexpr int NS = HD / 32, ND = HD / 16, NC = 16 * NT;
  constexpr int OS = HD + 4;  // LDS row stride (floats): 16 rows fall in different banks
  constexpr int ES = (int)sizeof(KT);
  __shared__ __align__(16) float s_o[4 * NC * OS];
  __shared__ float s_m[4 * NC], s_l[4 * NC];

  const unsigned item = blockIdx.x / (unsigned)a.hkv;
  const int kvh = (int)(blockIdx.x - item * a.hkv);
  const AttendSpan sp = a.sp[__builtin_amdgcn_readfirstlane(find_span(a, item))];
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  const int lc = l & 15, lg = l >> 4;
  const int ncol = sp.n * a.G, tiles = (ncol + NC - 1) / NC;
  const int local = (int)(item - sp.first), split = local / tiles, tile = local - split * tiles;
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
  auto load = [&](Pair& b, int pg) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int pid = ld_const<int>(bt + min(pg + x, p1 - 1));  // (past the run: its last page again)
      const size_t slot = ((size_t)a.layer * a.num_pages + pid) * a.hkv + kvh;
      const char* kb = (const char*)a.kpool + slot * (16 * HD * ES);
      const char* vb = (const char*)a.vpool + slot * (16 * HD * ES);
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int y = 0; y < KW; ++y)
          b.k[x][s][y] = __builtin_nontemporal_load((global_ptr<KRaw>)(kb + (s * 512 + 8 * l) * ES + 16 * y));
#pragma unroll
      for (int d = 0; d < ND; ++d) b.v[x][d] = __builtin_nontemporal_load((global_ptr<VRaw>)(vb + (d * 256 + 4 * l) * ES));
      if constexpr (I8) {
        b.ks[x] = ld_global<f32x4>((const char*)a.kpool + a.scales + slot * 64 + 16 * lg);
        b.vs[x] = ld_global<f32x4>((const char*)a.vpool + a.scales + slot * 64 + 16 * lg);
      }
    }
  };
  auto key = [&](const KRaw* raw, bf16x8* k) {
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
        split3(__uint_as_float(raw[i >> 1][2 * (i & 1)]), __uint_as_float(raw[i >> 1][2 * (i & 1) + 1]), s);
#pragma unroll
        for (int z = 0; z < 3; ++z) p[z][i] = s[z];
      }
#pragma unroll
      for (int z = 0; z < KP; ++z) k[z] = __builtin_bit_cast(bf16x8, p[z]);
    }
  };
  // dims 16 d + lc of positions 4 lg .. of both pages
  auto value = [&](const VRaw& va, const VRaw& vb, bf16x8* v) {
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
        split3(__uint_as_float(src[2 * (i & 1)]), __uint_as_float(src[2 * (i & 1) + 1]), s);
#pragma unroll
        for (int z = 0; z < 3; ++z) p[z][i] = s[z];
      }
#pragma unroll
      for (int z = 0; z < KP; ++z) v[z] = __builtin_bit_cast(bf16x8, p[z]);
    }
  };
  // products of parts i and j with i + j < 3 (the others are below 2^-24)
  auto mma = [&](const bf16x8* x, const bf16x8* y, f32x4 acc) {
#pragma unroll
    for (int i = KP - 1; i >= 0; --i)
#pragma unroll
      for (int j = PARTS - 1; j >= 0; --j)
        if (i + j < 3) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], y[j], acc, 0, 0, 0);
    return acc;
  };
  auto compute = [&](const Pair& b, int pg) {
    const bool whole = 16 * pg >= flo && 16 * pg + 32 <= fhi && pg + 1 < p1;  // (uniform)
    f32x4 s[NT][2];
#pragma unroll
    for (int u = 0; u < NT; ++u) s[u][0] = s[u][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        bf16x8 kk[KP];
        key(b.k[x][k], kk);
#pragma unroll
        for (int u = 0; u < NT; ++u) s[u][x] = mma(kk, q[u][k], s[u][x]);
      }
    bf16x8 p[NT][PARTS];
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
      const bool grow = mx > m[u] + kSlack;
      if (__ballot(grow)) {
        const float mn = grow ? mx : m[u];
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
      u32x4 pw[PARTS];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (PARTS == 1) {
          pw[0][i] = pk_bf16(pv[2 * i], pv[2 * i + 1]);
        } else {
          uint32_t s3[3];
          split3(pv[2 * i], pv[2 * i + 1], s3);
#pragma unroll
          for (int k = 0; k < PARTS; ++k) pw[k][i] = s3[k];
        }
      }
#pragma unroll
      for (int k = 0; k < PARTS; ++k) p[u][k] = __builtin_bit_cast(bf16x8, pw[k]);
    }
    bool odd = false;
    if (!I8 && !whole) {  // an infinite or NaN V anywhere in the pair?
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
        value(b.v[0][d], b.v[1][d], v);
#pragma unroll
        for (int u = 0; u < NT; ++u) o[u][d] = mma(v, p[u], o[u][d]);
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
          value(va, vb, v);
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            const f32x4 t = mma(v, p[u], o[u][d]);
            if (crow[u] == r) o[u][d] = t;
          }
        }
      }
    }
  };
  if (p0 < p1) {
    load(buf[0], p0);
    for (int pg = p0; pg < p1; pg += 4) {
      if (pg + 2 < p1) load(buf[1], pg + 2);
      compute(buf[0], pg);
      if (pg + 2 < p1) {
        if (pg + 4 < p1) load(buf[0], pg + 4);
        compute(buf[1], pg + 2);
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
      st_out4<IT>(a, sp.row0 + r, h, 4 * d4, acc * (L == 0.f ? 0.f : 1.f / L));
      if (d4 == 0 && a.lse != nullptr)
        a.lse[(size_t)(sp.row0 + r) * a.hq + h] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
    } else {
      const size_t part = sp.part0 + ((size_t)r * a.hq + h) * sp.nsplit + split;
      *(f32x4*)(a.part + part * HD + 4 * d4) = acc;
      if (d4 == 0) *(float2*)(a.ml + part * 2) = make_float2(M, L);
    }
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
  const AttendSpan sp = a.sp[__builtin_amdgcn_readfirstlane(find_span(a, item))];
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
  st_out4<IT>(a, sp.row0 + r, h, 4 * d4, Ot * (Lt == 0.f ? 0.f : 1.f / Lt));
  if (d4 == 0 && a.lse != nullptr)
    a.lse[(size_t)(sp.row0 + r) * a.hq + h] = Lt == 0.f ? -INFINITY : (Mt + __builtin_amdgcn_logf(Lt)) * kLn2;
}

template <class KT, class IT, int HD>
static hipError_t launch_kind(int kind, const AttendArgs& a, hipStream_t s) {
  const dim3 grid(a.n_items * (unsigned)a.hkv), block(256);
  if (kind == 0) return launch_k(k_attend_rows<KT, IT, HD, 1>, grid, block, s, a);
  return launch_k(k_attend_rows<KT, IT, HD, 2>, grid, block, s, a);
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

hipError_t launch_attend_merge(int io, int hd, const AttendArgs& a, hipStream_t s) {
  const dim3 grid(a.n_items), block(256);
  if (io == 1) return hd == 128 ? launch_k(k_attend_merge<bf16_t, 128>, grid, block, s, a) : launch_k(k_attend_merge<bf16_t, 64>, grid, block, s, a);
  return hd == 128 ? launch_k(k_attend_merge<float, 128>, grid, block, s, a) : launch_k(k_attend_merge<float, 64>, grid, block, s, a);
}

}  // namespace laser
