// Rows of K and V written into the paged cache and read out of it (laser_kv_write, laser_kv_read, and
// import / export of INT8 caches), and the quantisation of a forward's new rows.
//
// An INT8 cache holds, per (layer, position, kv head), s = amax / 127 in fp32 and the integers
// q = rint(127 x / amax) in -127 .. 127; it stands for q s.  127 x is exact for bf16 rows, so a value
// half way between two steps is seen as such (x = amax / 2 is common) and goes to the even one.  A row
// with a NaN or an infinity gets that as its scale and zeros: all of it reads back as NaN.
//
// Both are bounded by memory: a row of 128 bf16 dims is 256 bytes in, 132 out.  A thread takes 4
// positions (those that share the V block's groups of 4) x 8 dims of K or of V, as the page blocks want
// them: 8 dims of a position are contiguous in a K block, 4 positions of a dim in a V block, so that
// every access is of 8 to 32 bytes; the hd / 8 lanes of a row find its amax without LDS.  A workgroup
// belongs to one run of rows, whose page ids it looks up.
//
// Measured within a graph, 14,336 bf16 rows of 8 heads x 128, bytes read and written: into INT8 19.4 us (4.6 TB/s),
// bf16 29.6 us (4.0), E4M3 17.5 us (5.0); out of INT8 20.1 us (4.4), bf16 24.5 us (4.8), E4M3 20.1 us (4.4).  A copy of
// 1 GiB reaches 5.1 TB/s.  INT8 was bound by the quantisation's instructions: 23.8 us with a rounding, a clamp and a
// division per row and lane more.  A single row is latency: 3.5 us.
#include "device_common.hpp"
#include "kernels.hpp"

namespace laser {

namespace {

// Largest of v over the hd/8 lanes that hold a row.  (Absolute values as unsigned bits order like the
// floats, with infinity and NaN on top: a NaN is not lost.)
template <int LD8>
__device__ __forceinline__ uint32_t row_umax(uint32_t v) {
  auto dpp = [](uint32_t x, auto c) { return (uint32_t)__builtin_amdgcn_update_dpp(0u, x, decltype(c)::value, 0xf, 0xf, false); };
  v = max(v, dpp(v, std::integral_constant<int, kDppQuad1032>{}));
  v = max(v, dpp(v, std::integral_constant<int, kDppQuad2301>{}));
  v = max(v, dpp(v, std::integral_constant<int, kDppHalfMirror>{}));
  if (LD8 == 4) v = max(v, dpp(v, std::integral_constant<int, kDppRowRor8>{}));
  return v;
}

// Largest magnitude of 8 elements, as bits (a NaN is the largest).
__device__ __forceinline__ uint32_t amax8(const float* x) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) m = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, fabsf(x[e])), fabsf(x[e + 1]));
  return __float_as_uint(m) & 0x7fffffffu;
}

// A row's scale.
__device__ __forceinline__ float scale_of(uint32_t amax_bits) {
  const float amax = __uint_as_float(amax_bits);
  return amax_bits >= 0x7f800000u ? amax : amax / 127.f;
}

// What a row's elements are multiplied by and divided by: rows far from 1 are moved by a
// power of two first, so that neither 127 x nor 1 / amax leaves the normal range.
struct RowScale {
  float pre, top, inv, off0;
  __device__ __forceinline__ explicit RowScale(uint32_t amax_bits) {
    const float amax = __uint_as_float(amax_bits);
    const float c = amax > 0x1p100f ? 0x1p-32f : (amax < 0x1p-60f ? 0x1p64f : 1.f);
    pre = 127.f * c;
    top = amax * c;
    const bool small = amax < 0x1p-100f;  // (127 / amax may leave the range: divided)
    inv = amax_bits >= 0x7f800000u || amax == 0.f ? 0.f : small ? 1.f : pre * __builtin_amdgcn_rcpf(top);
    off0 = small ? 1.f : 0.f;
  }
  // rint(127 x / amax) of 8 elements in the low bytes of t.  The sum of a product with 127 / amax and 1.5 2^23 is rounded
  // to the integer by itself and has it in its low bits.  127 / amax from the 1-ulp reciprocal is off by less than
  // 2^-23 + 2^-24 of itself, a product by less than 2^-15 steps; only next to half a step does that matter, and then the
  // division decides.
  __device__ __forceinline__ void quant8(const float* x, uint32_t* t) const {
    constexpr float kInt = 0x1.8p23f;
    float off = off0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = __builtin_fmaf(x[e], inv, kInt);
      t[e] = __float_as_uint(y);
      off = fmaxf(off, fabsf(__builtin_fmaf(x[e], inv, kInt - y)));
    }
    if (off > 0.5f - 0x1p-15f)
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = (uint32_t)(int)rintf(x[e] * pre / top);
  }
  // What the integers of a row without a scale (zeros, NaN, infinities) are taken as: zeros.
  __device__ __forceinline__ uint32_t keep() const { return inv == 0.f ? 0u : ~0u; }
};

// The low bytes of four words.
__device__ __forceinline__ uint32_t low4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(b, a, 0x0c0c0400u) | __builtin_amdgcn_perm(d, c, 0x04000c0cu);
}

// Four values as E4M3 (to nearest even, saturated at +-448; NaN stays NaN).
__device__ __forceinline__ uint32_t pk_fp8x4(const float* x) {
  float c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = x[i] != x[i] ? x[i] : fminf(fmaxf(x[i], -448.f), 448.f);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false), true);
}

__device__ __forceinline__ uint16_t f2bf_any(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

// 8 elements of one position in the cache's type.
template <class KT>
struct Piece {
  static constexpr int W = 2 * (int)sizeof(KT);  // words
  uint32_t w[W];
};
template <class KT>
__device__ __forceinline__ Piece<KT> pack(const float* x, const RowScale* rs) {
  Piece<KT> p;
  if constexpr (std::is_same_v<KT, float>) {
#pragma unroll
    for (int e = 0; e < 8; ++e) p.w[e] = __float_as_uint(x[e]);
  } else if constexpr (std::is_same_v<KT, bf16_t>) {
#pragma unroll
    for (int e = 0; e < 4; ++e) p.w[e] = (uint32_t)f2bf_any(x[2 * e]) | ((uint32_t)f2bf_any(x[2 * e + 1]) << 16);
  } else {
    if constexpr (std::is_same_v<KT, fp8_t>) {
      p.w[0] = pk_fp8x4(x);
      p.w[1] = pk_fp8x4(x + 4);
    } else {
      uint32_t t[8];
      rs->quant8(x, t);
#pragma unroll
      for (int h = 0; h < 2; ++h) p.w[h] = low4(t[4 * h], t[4 * h + 1], t[4 * h + 2], t[4 * h + 3]) & rs->keep();
    }
  }
  return p;
}
template <class KT>
__device__ __forceinline__ void unpack(const Piece<KT>& p, float scale, float* x) {
  if constexpr (std::is_same_v<KT, float>) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(p.w[e]);
  } else if constexpr (std::is_same_v<KT, bf16_t>) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float((e & 1) ? (p.w[e >> 1] & 0xffff0000u) : (p.w[e >> 1] << 16));
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (std::is_same_v<KT, fp8_t>) {
        uint32_t lo, hi;
        fp8x4_to_bf16x4(p.w[h], lo, hi);
        x[4 * h + 0] = __uint_as_float(lo << 16);
        x[4 * h + 1] = __uint_as_float(lo & 0xffff0000u);
        x[4 * h + 2] = __uint_as_float(hi << 16);
        x[4 * h + 3] = __uint_as_float(hi & 0xffff0000u);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * h + e] = (float)(int)(int8_t)(p.w[h] >> (8 * e)) * scale;
      }
    }
  }
}

// Element e of a piece, as stored bits; and put back.
template <class KT>
__device__ __forceinline__ uint32_t get_e(const uint32_t* w, int e) {
  if constexpr (sizeof(KT) == 4) return w[e];
  if constexpr (sizeof(KT) == 2) return (w[e >> 1] >> (16 * (e & 1))) & 0xffffu;
  return (w[e >> 2] >> (8 * (e & 3))) & 0xffu;
}
template <class KT>
__device__ __forceinline__ void put_e(uint32_t* w, int e, uint32_t v) {
  if constexpr (sizeof(KT) == 4) w[e] = v;
  if constexpr (sizeof(KT) == 2) w[e >> 1] |= v << (16 * (e & 1));
  if constexpr (sizeof(KT) == 1) w[e >> 2] |= v << (8 * (e & 3));
}

template <class KT>
__device__ __forceinline__ void ld_words(const char* p, uint32_t* w) {
  constexpr int W = Piece<KT>::W;
  if constexpr (W == 2) {
    const u32x2 v = ld_global<u32x2>(p);
    w[0] = v[0];
    w[1] = v[1];
  } else {
#pragma unroll
    for (int q = 0; q < W / 4; ++q) {
      const u32x4 v = ld_global<u32x4>(p + 16 * q);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[4 * q + i] = v[i];
    }
  }
}
template <class KT>
__device__ __forceinline__ void st_words(char* p, const uint32_t* w) {
  constexpr int W = Piece<KT>::W;
  if constexpr (W == 2) {
    *(u32x2*)p = u32x2{w[0], w[1]};
  } else {
#pragma unroll
    for (int q = 0; q < W / 4; ++q) *(u32x4*)(p + 16 * q) = u32x4{w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]};
  }
}

// 8 elements of a caller's row (VEC: 16-byte aligned pieces).  Rows of 16 bits are read non-temporally, so
// that the block lines under assembly stay (14,336 rows x 8 heads x 128 into E4M3: 17.5 us, 18.9 without); in fp32 a
// lane's two loads share lines, and it costs (8,000 rows x 4 heads x 128, INT8: 7% more).
template <class IT, bool VEC>
__device__ __forceinline__ void ld_row8(const void* base, int64_t e, float* x) {
  if constexpr (VEC) {
    Piece<IT> p;
    const char* at = (const char*)base + e * (int64_t)sizeof(IT);
    if constexpr (Piece<IT>::W == 4) {
      const u32x4 v = ld_nt16(at);
#pragma unroll
      for (int i = 0; i < 4; ++i) p.w[i] = v[i];
    } else {
      ld_words<IT>(at, p.w);
    }
    unpack<IT>(p, 0.f, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = ldw<IT>(base, (size_t)(e + i));
  }
}
template <class IT, bool VEC>
__device__ __forceinline__ void st_row8(void* base, int64_t e, const float* x) {
  const Piece<IT> p = pack<IT>(x, nullptr);
  if constexpr (VEC) {
    st_words<IT>((char*)base + e * (int64_t)sizeof(IT), p.w);
  } else {
    using E = std::conditional_t<sizeof(IT) == 2, uint16_t, uint32_t>;
#pragma unroll
    for (int i = 0; i < 8; ++i) ((E*)base)[e + i] = (E)get_e<IT>(p.w, i);
  }
}

}  // namespace

// grid (workgroups of all runs, layers, K and V), 256 threads: thread -> (page, kv head, 4 positions, 8 dims), so
// that a wave writes whole page blocks.
template <class KT, class IT, int LD8, bool WRITE, bool VEC>
__global__ __launch_bounds__(256) void k_kv_rows(KvRowsArgs a) {
  constexpr int HD = 8 << LD8;
  const int lane = threadIdx.x & 63;
  // the run: the last one that starts at or before this workgroup
  const unsigned first = lane < a.n_runs ? a.runs[lane].first : 0xffffffffu;
  const int ri = __builtin_popcountll(__ballot(first <= blockIdx.x)) - 1;
  const KvRun run = a.runs[ri];
  const unsigned idx = (blockIdx.x - run.first) * 256 + threadIdx.x;
  const int d8 = idx & ((1 << LD8) - 1);
  const unsigned r = idx >> (LD8 + 2), g = r / (unsigned)a.hkv;
  const int kvh = (int)(r - g * a.hkv);
  const int pos4 = 4 * ((run.pos >> 4) + (int)g) + ((idx >> LD8) & 3);  // group of 4 positions
  const int lo = max(run.pos - 4 * pos4, 0), hi = min(run.pos + run.n - 4 * pos4, 4);  // the run's part of it
  if (hi <= lo) return;  // (whole rows of lanes leave together)
  const bool is_v = blockIdx.z;
  const int layer = a.layer + blockIdx.y;
  const int page = a.bt[(size_t)run.seq * a.max_pps + (pos4 >> 2)], t4 = pos4 & 3;
  const size_t slot = ((size_t)layer * a.num_pages + page) * a.hkv + kvh;
  char* pool = (char*)(is_v ? a.vpool : a.kpool);
  char* blk = pool + (slot * (16 * HD) + (is_v ? v_block_off(4 * t4, 8 * d8) : k_block_off(4 * t4, 8 * d8))) * sizeof(KT);
  float* sc = (float*)(pool + a.scales) + slot * 16 + 4 * t4;  // (INT8)
  void* dense = is_v ? a.v : a.k;
  const int64_t row_stride = is_v ? a.v_row : a.k_row;
  const int64_t e0 = (int64_t)blockIdx.y * (is_v ? a.v_layer : a.k_layer) + kvh * (is_v ? a.v_head : a.k_head) + 8 * d8 +
                     (run.row0 + 4 * (int64_t)pos4 - run.pos) * row_stride;  // of the group's position 0 (maybe before the run)
  float x[4][8];
  if constexpr (WRITE) {
    Piece<KT> p[4];
    [[maybe_unused]] uint32_t t8[4][8], keep = 0, mine = 0;  // INT8: the integers; bytes that stay; row d8 % 4's maximum
#pragma unroll
    for (int j = 0; j < 4; ++j) ld_row8<IT, VEC>(dense, e0 + min(max(j, lo), hi - 1) * row_stride, x[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (std::is_same_v<KT, i8_t>) {
        const uint32_t amax = row_umax<LD8>(amax8(x[j]));
        const RowScale rs(amax);
        if ((d8 & 3) == j) mine = amax;
        rs.quant8(x[j], t8[j]);
#pragma unroll
        for (int h = 0; h < 2; ++h) p[j].w[h] = low4(t8[j][4 * h], t8[j][4 * h + 1], t8[j][4 * h + 2], t8[j][4 * h + 3]) & rs.keep();
        keep |= rs.keep() & (0xffu << (8 * j));
      } else {
        p[j] = pack<KT>(x[j], nullptr);
      }
    }
    if constexpr (std::is_same_v<KT, i8_t>)  // (each lane one row's scale: a division is ten instructions)
      if (d8 < 4 && d8 >= lo && d8 < hi) sc[d8] = scale_of(mine);
    if (hi - lo == 4) {  // 32 elements: 8 e + j of a K block (dim j, position e), 4 e + j of a V block (position j, dim e)
      uint32_t t[4 * Piece<KT>::W] = {};
      if (!is_v) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < Piece<KT>::W; ++e) t[j * Piece<KT>::W + e] = p[j].w[e];
      } else if constexpr (std::is_same_v<KT, i8_t>) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = low4(t8[0][e], t8[1][e], t8[2][e], t8[3][e]) & keep;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j) put_e<KT>(t, 4 * e + j, get_e<KT>(p[j].w, e));
      }
#pragma unroll
      for (int q = 0; q < Piece<KT>::W; ++q) *(u32x4*)(blk + 16 * q) = u32x4{t[4 * q], t[4 * q + 1], t[4 * q + 2], t[4 * q + 3]};
    } else if (!is_v) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j >= lo && j < hi) st_words<KT>(blk + j * 8 * sizeof(KT), p[j].w);
    } else {  // (the group's other positions keep what they hold)
      using E = std::conditional_t<sizeof(KT) == 1, uint8_t, std::conditional_t<sizeof(KT) == 2, uint16_t, uint32_t>>;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j >= lo && j < hi)
#pragma unroll
          for (int e = 0; e < 8; ++e) ((E*)blk)[4 * e + j] = (E)get_e<KT>(p[j].w, e);
    }
  } else {
    uint32_t w[4 * Piece<KT>::W];
#pragma unroll
    for (int q = 0; q < Piece<KT>::W; ++q) {
      const u32x4 x = ld_global<u32x4>(blk + 16 * q);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[4 * q + i] = x[i];
    }
    f32x4 s4 = {1.f, 1.f, 1.f, 1.f};
    if constexpr (std::is_same_v<KT, i8_t>) s4 = ld_global<f32x4>(sc);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      Piece<KT> p{};
      if (is_v) {
#pragma unroll
        for (int e = 0; e < 8; ++e) put_e<KT>(p.w, e, get_e<KT>(w, 4 * e + j));
      } else {
#pragma unroll
        for (int e = 0; e < Piece<KT>::W; ++e) p.w[e] = w[j * Piece<KT>::W + e];
      }
      unpack<KT>(p, s4[j], x[j]);
      if (j >= lo && j < hi) st_row8<IT, VEC>(dense, e0 + j * row_stride, x[j]);
    }
  }
}

// A forward's rows: grid (rows, heads of K and of V), thread d8 of a head takes 8 dims.  Its two dependent reads
// (page id, row) and scattered stores of a few KB are latency: the 28 launches of a 7B decode step (batch 1 behind
// 14,336 positions) take about 70 of its 2,777 us.
template <int LD8>
__global__ __launch_bounds__(256) void k_kv_quant(const Plan* plan, const float* rows, void* kpool, void* vpool, size_t scales,
                                                  const int* bt, int max_pps, int num_pages, int layer, int hkv) {
  constexpr int HD = 8 << LD8;
  const int m = blockIdx.x, idx = blockIdx.y * 256 + threadIdx.x;
  const int d8 = idx & ((1 << LD8) - 1), kh = idx >> LD8;  // kh: K heads, then V heads
  if (kh >= 2 * hkv) return;  // (whole rows of lanes leave together)
  float x[8];
  ld_row8<float, true>(rows, ((int64_t)m * 2 * hkv + kh) * HD + 8 * d8, x);
  const RowDesc rd = row_desc(plan, m);
  const int page = bt[(size_t)rd.seq * max_pps + (rd.pos >> 4)], t = rd.pos & 15;
  const uint32_t amax = row_umax<LD8>(amax8(x));
  const RowScale rs(amax);
  const Piece<i8_t> p = pack<i8_t>(x, &rs);
  const bool is_v = kh >= hkv;
  char* pool = (char*)(is_v ? vpool : kpool);
  const size_t slot = ((size_t)layer * num_pages + page) * hkv + (is_v ? kh - hkv : kh);
  char* blk = pool + slot * (16 * HD) + (is_v ? v_block_off(t, 8 * d8) : k_block_off(t, 8 * d8));
  if (is_v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) blk[4 * e] = (char)get_e<i8_t>(p.w, e);
  } else {
    st_words<i8_t>(blk, p.w);
  }
  if (d8 == 0) ((float*)(pool + scales))[slot * 16 + t] = scale_of(amax);
}

hipError_t launch_kv_quant(const Plan* plan, int M, const float* rows, void* kpool, void* vpool, size_t scales, const int* bt,
                           int max_pps, int num_pages, int layer, int hkv, int hd, hipStream_t s) {
  if (M < 1 || (hd != 64 && hd != 128)) return hipErrorInvalidValue;
  const dim3 grid(M, (2 * hkv * (hd / 8) + 255) / 256), block(256);
  if (hd == 128)
    return launch_k(k_kv_quant<4>, grid, block, s, plan, rows, kpool, vpool, scales, bt, max_pps, num_pages, layer, hkv);
  return launch_k(k_kv_quant<3>, grid, block, s, plan, rows, kpool, vpool, scales, bt, max_pps, num_pages, layer, hkv);
}

template <class KT, class IT, int LD8>
static hipError_t launch_rows(const KvRowsArgs& a, bool write, bool vec, dim3 grid, hipStream_t s) {
  const dim3 block(256);
  if (write)
    return vec ? launch_k(k_kv_rows<KT, IT, LD8, true, true>, grid, block, s, a)
               : launch_k(k_kv_rows<KT, IT, LD8, true, false>, grid, block, s, a);
  return vec ? launch_k(k_kv_rows<KT, IT, LD8, false, true>, grid, block, s, a)
             : launch_k(k_kv_rows<KT, IT, LD8, false, false>, grid, block, s, a);
}

hipError_t launch_kv_rows(int kv_type, int io, int hd, KvRowsArgs& a, int n_layers, bool write, hipStream_t s) {
  if (a.n_runs < 1 || a.n_runs > kKvRuns || n_layers < 1 || n_layers > 65535 || (hd != 64 && hd != 128)) return hipErrorInvalidValue;
  unsigned wgs = 0;
  for (int i = 0; i < a.n_runs; ++i) {
    KvRun& r = a.runs[i];
    if (r.n < 1) return hipErrorInvalidValue;
    const unsigned pages = (unsigned)((r.pos + r.n + kPage - 1) / kPage - r.pos / kPage);
    r.first = wgs;
    wgs += (unsigned)(((uint64_t)pages * a.hkv * (hd / 2) + 255) / 256);
  }
  const int es = io == 1 ? 2 : 4;
  auto on16 = [&](int64_t e) { return e * es % 16 == 0; };
  if ((((uintptr_t)a.kpool | (uintptr_t)a.vpool) & 15) != 0) return hipErrorInvalidValue;
  const bool vec = ((((uintptr_t)a.k | (uintptr_t)a.v) & 15) == 0) && on16(a.k_row) && on16(a.k_head) && on16(a.k_layer) && on16(a.v_row) && on16(a.v_head) && on16(a.v_layer);
  const dim3 grid(wgs, n_layers, 2);
  auto go = [&](auto kt) {
    using KT = decltype(kt);
    if (io == 1) return hd == 128 ? launch_rows<KT, bf16_t, 4>(a, write, vec, grid, s) : launch_rows<KT, bf16_t, 3>(a, write, vec, grid, s);
    return hd == 128 ? launch_rows<KT, float, 4>(a, write, vec, grid, s) : launch_rows<KT, float, 3>(a, write, vec, grid, s);
  };
  switch (kv_type) {
    case 0: return go(float{});
    case 1: return go(bf16_t{});
    case 2: return go(fp8_t{});
    default: return go(i8_t{});
  }
}

}  // namespace laser
