// Dense attention: what its kernels share.  Arguments, LDS tiles of 32 token
// rows and their MFMA operands, score variants, masks.
//
// Every kernel works on pairs of a "streamed" tile of 32 rows in LDS and 32
// "held" rows of a wavefront in registers: scores of the pair come as the C
// layout of a 32 x 32 MFMA with one held row per lane (column l % 32) and the
// streamed rows 8 b + 4 (l / 32) + r in register 4 b + r.  Rounded to the
// operand type, registers 8 kp .. 8 kp + 7 are the B operand of a product over
// the streamed rows as they are, when the A operand (read transposed from the
// same LDS tile) takes the rows in that order.
//
// Query rows of one key/value head are packed: row r = i G + g is query i of
// the head's g-th query head, so that heads that share keys share their tiles.
#pragma once

#include "attn_tile.h"
#include "common.h"

namespace park {

typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef short i16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));

struct fp8_t {  // a cached value: e4m3 with the power of two of its page and head
  uint8_t x;
};

struct RowsArg {  // [B][H][N][d] view, strides in bytes
  char* p;
  int64_t b, h, r;
};

// document ids of 32 consecutive rows: smallest and largest id that is not
// negative, and whether all 32 are one such id
struct DocTile {
  int lo, hi, uni, pad;
};
// ids [B][N] of packed rows r = i G + g and where their tiles' go
struct DocIds {
  const int* ids;
  int N, G;
  DocTile* out;
  __host__ __device__ int tiles() const { return (int)(((int64_t)N * G + 31) / 32); }
};

// How the tiles of held rows become workgroups: the first `whole` tiles one
// each, the other `rest` as n each, which take parts of the streamed rows and
// leave partial sums of ROWS rows, at part[(s rest + tile - whole) ROWS ..].
struct DenseSplit {
  int whole, rest, n;
  int64_t groups() const { return whole + (int64_t)rest * n; }
  __host__ __device__ size_t rows(int held) const { return (size_t)rest * n * held; }
};

struct DenseArgs {
  RowsArg q, k, v, o;
  int B, Hkv, G, Nq, Nk, R;  // R = Nq G packed rows of a key/value head
  uint32_t gmul;             // r / G = (r gmul) >> (31 + gshift) for r < 2^31 (G > 1)
  int gshift;
  int causal, q_pos;
  const int* prefix;          // [B] or null
  const int *q_doc, *k_doc;   // [B][Nq], [B][Nk] or null
  const DocTile* k_tiles;     // [B][ceil(Nk / 32)] (with documents)
  const float* slopes;        // [Hq] or null
  float scale, cap;           // cap = 0: none
  float cap_arg, cap_exp;     // scale / cap, and 2 log2(e) times that
  float cap_small;            // products below it: |scale s / cap| < 5/16
  float* lse;                 // [B][Hq][Nq] or null
  int out_f32;
  DenseSplit split;
  float* part;                // unnormalised sums of the split tiles' rows
  float2* ml;                 // their maxima and sums
  // cache (fp8_t): pools [n_pages][Hkv][page][D], exponents [n_pages][Hkv]
  const int8_t *k_exp, *v_exp;
  const int* table;           // [B][max_pages]
  const int *lens, *q_lens;   // [B] (q_lens may be null)
  int page_shift, n_pages, max_pages;
  int* status;                // may be null
};

// starting maximum of a row; scores below it count as -infinity (its product
// with the largest scale is finite, so that a masked score never meets an
// infinity of the other sign)
constexpr float DENSE_NOKEY = -1e30f;
constexpr int DENSE_ROWS = 128;                // held rows of a workgroup
constexpr int DENSE_PAGES = 2048;              // pages a workgroup of the cache kernel can hold
// range of the exponent of a cached page and head, which writing holds to and reading
// clamps to (448 2^119 is finite, and the smallest e4m3 value's 2^-119 normal, in bf16)
constexpr int CACHE_EMIN = -110, CACHE_EMAX = 119;
constexpr int DENSE_MAXSPLIT = 64;
constexpr int DENSE_FEW = 32;                  // rows of a head that its own form takes

// ------------------------------------------------------------------ LDS tiles
// 32 rows of D elements in blocks of 1 KB: 16 rows (r / 16 = block % 2) x 64
// bytes (column block / 2), a row's four 16-byte chunks XORed with (r / 4) % 4.
// A block is one wave-wide copy, four lanes to a row's 64 bytes.  Of the places
// a lane reads, as row operands or by transposed reads, all but one XOR lie at
// constant distances, so that a tile costs two address registers for each kind
// instead of one per read; 16 rows x 16 bytes, 4 rows x 64 bytes (bf16) and
// 8 rows x 32 bytes (e4m3) each cover the 64 banks once.
template <class T, int D>
struct DenseTile {
  static constexpr int ES = sizeof(T), BYTES = 32 * D * ES;
  static constexpr int NDMA = BYTES / 1024;         // copies per tile
  static constexpr int NI = (NDMA + 3) / 4;         // ... per wavefront
  static constexpr int DW = NDMA / NI;              // wavefronts that issue them
  // byte offset of element (row, col)
  static __device__ __forceinline__ uint32_t at(int row, int col) {
    const int byte = col * ES, c = byte >> 4;
    return 1024 * (2 * (c >> 2) + (row >> 4)) + 64 * (row & 15) +
           16 * ((c & 3) ^ ((row >> 2) & 3)) + (byte & 15);
  }
  // the part of block c that lane l copies: row and byte within the row
  static __device__ __forceinline__ int copy_row(int c, int l) { return 16 * (c & 1) + (l >> 2); }
  static __device__ __forceinline__ uint32_t copy_byte(int c, int l) {
    return 64 * (c >> 1) + 16 * ((l & 3) ^ ((l >> 4) & 3));
  }
  // where a lane reads row operands and transposed ones, from the tile's start
  static __device__ __forceinline__ uint32_t row_at(int l) { return at(l & 31, 8 * (l >> 5)); }
  static __device__ __forceinline__ uint32_t col_at(int l) {
    const int hf = l >> 5, G = (l >> 4) & 1, j = l & 15;
    if constexpr (ES == 4) return at(4 * hf, l & 31);
    // 16-lane group: lane j supplies row 4 hf + j / 4, columns 4 (j % 4) .. and
    // receives column j of 4 rows (a second read: the rows 8 further)
    else if constexpr (ES == 2) return at(4 * hf + (j >> 2), 16 * G + 4 * (j & 3));
    // lane j supplies row j / 2, columns 8 (j % 2) .. and receives column j of 8 rows
    else return at(4 * hf + ((j >> 1) & 3) + 8 * (j >> 3), 16 * G + 8 * (j & 1));
  }
};

// row of the k-th (0..7) streamed row of half hf in step kp of a product over
// the 32 streamed rows
__device__ __forceinline__ int dense_krow(int kp, int hf, int k) {
  return 16 * kp + 4 * hf + (k & 3) + 8 * (k >> 2);
}

// a wave-uniform value kept in a scalar register
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// x, without the compiler's knowledge of it: what is computed from it stays
// where it is written
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// e4m3 -> bf16 with the value's power of two (exact: 4 significant bits)
__device__ __forceinline__ uint32_t cvt_f8(uint32_t w, float s, bool hi) {
  return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true))
            : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
}
__device__ __forceinline__ bf16x8_t cvt_f8x8(u32x2_t w, float s) {
  return __builtin_bit_cast(bf16x8_t, make_uint4(cvt_f8(w[0], s, false), cvt_f8(w[0], s, true),
                                                 cvt_f8(w[1], s, false), cvt_f8(w[1], s, true)));
}

// operand type of the products: bf16 (also for e4m3 tiles) or float
// as it is used (frag) and as it is read from LDS (raw)
template <class T>
struct DenseOp {
  typedef bf16x8_t frag, raw;
};
template <>
struct DenseOp<fp8_t> {
  typedef bf16x8_t frag;
  typedef u32x2_t raw;
};
template <>
struct DenseOp<float> {
  typedef f32x8_t frag, raw;
};
template <class T>
__device__ __forceinline__ typename DenseOp<T>::frag dense_cvt(typename DenseOp<T>::raw f, float e) {
  if constexpr (sizeof(T) == 1) return cvt_f8x8(f, e);
  else return f;
}

__device__ __forceinline__ f32x16_t dense_mma(bf16x8_t a, bf16x8_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// eight steps of two: step e takes element e of both halves
__device__ __forceinline__ f32x16_t dense_mma(f32x8_t a, f32x8_t b, f32x16_t c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// 8 elements of a row in global memory as an operand (dims 16 s + 8 hf ..)
__device__ __forceinline__ void dense_load(bf16x8_t& f, const char* p) { f = *(const bf16x8_t*)p; }
__device__ __forceinline__ void dense_load(f32x8_t& f, const char* p) {
  const f32x4_t a = *(const f32x4_t*)p, b = *(const f32x4_t*)(p + 16);
  f = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// waits for an operand's loads
__device__ __forceinline__ void dense_arrived(const bf16x8_t& f) { asm volatile("" ::"v"(f)); }
__device__ __forceinline__ void dense_arrived(const f32x8_t& f) {
  asm volatile("" ::"v"(__builtin_shufflevector(f, f, 0, 1, 2, 3)),
               "v"(__builtin_shufflevector(f, f, 4, 5, 6, 7)));
}

// A operand, streamed row l % 32, dims 16 s + 8 hf .. + 7; base: tile + row_at(l)
template <class T, int D>
__device__ __forceinline__ typename DenseOp<T>::raw dense_row_raw(uint32_t base, int s) {
  if constexpr (sizeof(T) == 4) {
    const f32x4_t a = *(lds_f32x4_t*)(base + 2048 * s);
    const f32x4_t b = *(lds_f32x4_t*)((base ^ 16) + 2048 * s);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  } else if constexpr (sizeof(T) == 2) {
    return *(lds_bf16x8_t*)((base ^ (32 * (s & 1))) + 2048 * (s >> 1));
  } else {
    typedef const __attribute__((address_space(3))) u32x2_t lds_u2;
    return *(lds_u2*)((base ^ (16 * (s & 3))) + 2048 * (s >> 2));
  }
}

// A operand of a product over the streamed rows: column 32 db + l % 32, rows
// dense_krow(kp, hf, 0..7), by transposed LDS reads; base: tile + col_at(l)
template <class T, int D>
__device__ __forceinline__ typename DenseOp<T>::raw dense_col_raw(uint32_t base, int kp, int db) {
  if constexpr (sizeof(T) == 4) {
    f32x8_t f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      f[e] = *(const __attribute__((address_space(3))) float*)(
          (base ^ (32 * (e >> 2))) + 64 * (e & 3) + 512 * (e >> 2) + 1024 * kp + 4096 * db);
    return f;
  } else if constexpr (sizeof(T) == 2) {
    const uint32_t x = base + 1024 * kp + 2048 * db, y = (base ^ 32) + 512 + 1024 * kp + 2048 * db;
    const i16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)x);
    const i16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)y);
    return __builtin_bit_cast(bf16x8_t,
                              (i16x8_t)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    typedef __attribute__((address_space(3))) i32x2_t lds_i2;
    const uint32_t x = (base ^ (32 * (db & 1))) + 1024 * kp + 2048 * (db >> 1);
    return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2*)x));
  }
}

// scores (or their gradients) 8 kp .. 8 kp + 7 as an operand: bf16 by round to
// nearest even, float as they are
__device__ __forceinline__ void dense_pack(bf16x8_t& f, const f32x16_t& s, int kp) {
  uint4 u;
  u.x = pack_bf(s[8 * kp], s[8 * kp + 1]);
  u.y = pack_bf(s[8 * kp + 2], s[8 * kp + 3]);
  u.z = pack_bf(s[8 * kp + 4], s[8 * kp + 5]);
  u.w = pack_bf(s[8 * kp + 6], s[8 * kp + 7]);
  f = __builtin_bit_cast(bf16x8_t, u);
}
__device__ __forceinline__ void dense_pack(f32x8_t& f, const f32x16_t& s, int kp) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = s[8 * kp + e];
}

// Values that are not finite in a tile with masked pairs: they belong to the
// rows that allow their key and to no other, but 0 x NaN is NaN.  So they are
// taken out of the product, and counted by a product of their own: 1 for
// infinity, 2^8 for -infinity, 2^16 for NaN, times 1 for allowed pairs (sums of
// 32 are exact); what was counted is added to the row's sum.  All of it on
// integer arithmetic: comparisons would hold a scalar pair each.
//
// In each half (or word) of the words of an operand: 1 if it is not finite
__device__ __forceinline__ uint32_t odd_pair(uint32_t w) {
  return (((w & 0x7f807f80u) + 0x00800080u) >> 15) & 0x00010001u;
}
__device__ __forceinline__ uint32_t odd_word(uint32_t w) { return ((w & 0x7f800000u) + 0x00800000u) >> 31; }
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x8_t __attribute__((ext_vector_type(8)));

// nonzero if an operand holds a value that is not finite
__device__ __forceinline__ uint32_t dense_bad(bf16x8_t f) {
  const u32x4_t u = __builtin_bit_cast(u32x4_t, f);
  return odd_pair(u[0]) | odd_pair(u[1]) | odd_pair(u[2]) | odd_pair(u[3]);
}
__device__ __forceinline__ uint32_t dense_bad(f32x8_t f) {
  const u32x8_t u = __builtin_bit_cast(u32x8_t, f);
  uint32_t m = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) m |= odd_word(u[e]);
  return m;
}
// the operand with 0 for such values
__device__ __forceinline__ void dense_fix(bf16x8_t& f) {
  u32x4_t u = __builtin_bit_cast(u32x4_t, f);
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] &= ~(odd_pair(u[e]) * 0xffffu);
  f = __builtin_bit_cast(bf16x8_t, u);
}
__device__ __forceinline__ void dense_fix(f32x8_t& f) {
  u32x8_t u = __builtin_bit_cast(u32x8_t, f);
#pragma unroll
  for (int e = 0; e < 8; ++e) u[e] &= odd_word(u[e]) - 1u;
  f = __builtin_bit_cast(f32x8_t, u);
}
// the operand of their counts: 1, 2^8 or 2^16
__device__ __forceinline__ bf16x8_t dense_flag(bf16x8_t f) {
  u32x4_t u = __builtin_bit_cast(u32x4_t, f);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t m = odd_pair(u[e]), nan = (((u[e] & 0x007f007fu) + 0x007f007fu) >> 7) & m;
    u[e] = m * 0x3f80u + ((u[e] >> 15) & m & ~nan) * 0x400u + nan * 0x800u;
  }
  return __builtin_bit_cast(bf16x8_t, u);
}
__device__ __forceinline__ f32x8_t dense_flag(f32x8_t f) {
  u32x8_t u = __builtin_bit_cast(u32x8_t, f);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t m = odd_word(u[e]), nan = (((u[e] & 0x7fffffu) + 0x7fffffu) >> 23) & m;
    u[e] = m * 0x3f800000u + ((u[e] >> 31) & m & ~nan) * 0x04000000u + nan * 0x08000000u;
  }
  return __builtin_bit_cast(f32x8_t, u);
}
// bits 8 kp .. 8 kp + 7 as an operand of ones
__device__ __forceinline__ void dense_ones(bf16x8_t& f, uint32_t bits, int kp) {
  u32x4_t u;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t y = bits >> (8 * kp + 2 * e);
    u[e] = (y & 1u) * 0x3f80u + ((y >> 1) & 1u) * 0x3f800000u;
  }
  f = __builtin_bit_cast(bf16x8_t, u);
}
__device__ __forceinline__ void dense_ones(f32x8_t& f, uint32_t bits, int kp) {
  u32x8_t u;
#pragma unroll
  for (int e = 0; e < 8; ++e) u[e] = ((bits >> (8 * kp + e)) & 1u) * 0x3f800000u;
  f = __builtin_bit_cast(f32x8_t, u);
}
// ... for the operands f of one block of 32 columns and its sums
template <class frag>
__device__ __forceinline__ void dense_guard(frag (&f)[2], uint32_t ok, f32x16_t& acc) {
  if (!__any((dense_bad(f[0]) | dense_bad(f[1])) != 0u)) return;
  f32x16_t n = {};
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    frag one;
    dense_ones(one, ok, kk);
    n = dense_mma(dense_flag(f[kk]), one, n);
    dense_fix(f[kk]);
  }
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    const uint32_t c = (uint32_t)n[q];
    acc[q] += __uint_as_float((((c & 0xffu) + 0xffu) >> 8) * 0x7f800000u);
    acc[q] -= __uint_as_float(((((c >> 8) & 0xffu) + 0xffu) >> 8) * 0x7f800000u);
    acc[q] += __uint_as_float((((c >> 16) + 0xffffu) >> 16) * 0x7fc00000u);
  }
}

// bit q of a mask of pairs as a score (-infinity) or a summand (0) keeps or loses it
__device__ __forceinline__ float mask_score(float x, uint32_t bits, int q) {
  const uint32_t m = (uint32_t)((int)(bits << (31 - q)) >> 31);
  return __uint_as_float((__float_as_uint(x) & m) | (0xff800000u & ~m));
}
__device__ __forceinline__ float mask_zero(float x, uint32_t bits, int q) {
  return __uint_as_float(__float_as_uint(x) & (uint32_t)((int)(bits << (31 - q)) >> 31));
}
// 1 if x >= 0; 1 if x != 0
__device__ __forceinline__ uint32_t bit_ge0(int x) { return ~(uint32_t)x >> 31; }
__device__ __forceinline__ uint32_t bit_ne0(int x) { return (uint32_t)(x | -x) >> 31; }

// ------------------------------------------------------------- score variants
// The tanh cap of a tile's scores, c = cap tanh(x) with x = scale s / cap, and with
// GATE its derivative 1 - tanh^2.  Where |x| < 5/16, tanh is x (1 + z p(z)), z = x^2,
// with p of three terms fitted over that range (1.7e-8 off, relative); elsewhere it
// is 1 - 2 r with r = 1 / (1 + e^2x), whose derivative is 4 r (1 - r) and whose error,
// about 1e-7, is absolute: of a small score under a large cap it would leave little.
// So each element chooses for itself, also because a masked score, or another row's,
// is not to change a bit of it.  Scores are mostly small beside the cap: where all of
// a wavefront's are, the second form is left out (16 causal bf16 heads of 4096 rows,
// d = 64: 109 us at cap 50, 139 at cap 3, where no tile can; the gradient 306 and 375).
__device__ __forceinline__ float tanh_small(float x) {
  const float z = x * x;
  float p = fmaf(z, -0.0500828841f, 0.133117658f);
  p = fmaf(z, p, -0.333329902f);
  return fmaf(z * p, x, x);
}
// (of one score s)
__device__ __forceinline__ float dense_tanh(float s, const DenseArgs& a) {
  if (fabsf(s) < a.cap_small) return tanh_small(s * a.cap_arg);
  return fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s * a.cap_exp)), 1.0f);
}
template <bool GATE>
__device__ __forceinline__ void dense_cap_tile(f32x16_t& st, const DenseArgs& a, f32x16_t* gate) {
  float top = 0.0f;
#pragma unroll
  for (int q = 0; q < 16; ++q) top = fmaxf(top, fabsf(st[q]));
  if (!__any(!(top < a.cap_small))) {
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const float t = tanh_small(st[q] * a.cap_arg);
      st[q] = a.cap * t;
      if constexpr (GATE) (*gate)[q] = fmaf(-t, t, 1.0f);
    }
  } else {
    // (a number of its own: what both branches compute would be moved before them,
    // where it spills registers)
    float arg = a.cap_arg;
    asm volatile("" : "+s"(arg));
    // (both forms, then the choice: the compiler would branch for each element)
    auto choose = [](bool first, float x, float y) {
      asm("" : "+v"(x), "+v"(y));
      return first ? x : y;
    };
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const float t = tanh_small(st[q] * arg);
      const float r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(st[q] * a.cap_exp));
      const bool small = fabsf(st[q]) < a.cap_small;
      st[q] = choose(small, a.cap * t, fmaf(-2.0f * a.cap, r, a.cap));
      if constexpr (GATE) (*gate)[q] = choose(small, fmaf(-t, t, 1.0f), fmaf(-4.0f * r, r, 4.0f * r));
    }
  }
}

// This workgroup's tile of held rows and its part (-1: the whole).  Tiles of one
// head are side by side, so that those that run together read the same streamed
// rows; with a causal mask tiles of one place are, the longest first.
struct DenseItem {
  int head, tile, part, slot;  // slot: of the partial sums, in rows / held rows
};
__device__ __forceinline__ DenseItem dense_item(const DenseSplit& sp, int heads, int tiles, bool causal,
                                                bool last_first, int item) {
  DenseItem it = {0, 0, -1, 0};
  int unit = item;
  if (item >= sp.whole) {
    const int k = item - sp.whole;
    unit = sp.whole + k / sp.n;
    it.part = uniform(k % sp.n);
    it.slot = uniform(it.part * sp.rest + unit - sp.whole);
  }
  it.head = uniform(causal ? unit % heads : unit / tiles);
  const int t = causal ? unit / heads : unit % tiles;
  it.tile = uniform(last_first ? tiles - 1 - t : t);
  return it;
}
// part `i` of n of the streamed tiles [tbeg, tend)
__device__ __forceinline__ void dense_part(int i, int n, int& tbeg, int& tend) {
  const int share = (max(tend - tbeg, 0) + n - 1) / n;
  tbeg += i * share;
  tend = min(tend, tbeg + share);
}

// smallest lo and largest hi of a workgroup of NW wavefronts
template <int NW>
__device__ __forceinline__ void wg_range(int& lo, int& hi, int* red) {
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor(lo, o, 64));
    hi = max(hi, __shfl_xor(hi, o, 64));
  }
  __syncthreads();
  if (l == 0) {
    red[w] = lo;
    red[NW + w] = hi;
  }
  __syncthreads();
  lo = red[0];
  hi = red[NW];
#pragma unroll
  for (int i = 1; i < NW; ++i) {
    lo = min(lo, red[i]);
    hi = max(hi, red[NW + i]);
  }
}

// first and last 32-row tile in [0, n) whose document ids overlap [lo, hi]
// (n and -1: none)
template <int NW>
__device__ __forceinline__ void doc_range(const DocTile* tiles, int n, int lo, int hi, int* red,
                                          int& first, int& last) {
  first = n;
  last = -1;
  for (int t = threadIdx.x; t < n; t += 64 * NW)
    if (tiles[t].lo <= hi && tiles[t].hi >= lo) {
      first = min(first, t);
      last = t;
    }
  wg_range<NW>(first, last, red);
}

// The tiles of [tbeg, tend) whose rows are all of document `id` as one run
// [first, end) (empty if they are none or not one run); a wavefront's own
__device__ __forceinline__ void doc_run(const DocTile* tiles, int tbeg, int tend, int id, int& first,
                                        int& end) {
  int last = -1, count = 0;
  first = tend;
  for (int t = tbeg + (threadIdx.x & 63); t < tend; t += 64)
    if (tiles[t].uni && tiles[t].lo == id) {
      first = min(first, t);
      last = t;
      ++count;
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    first = min(first, __shfl_xor(first, o, 64));
    last = max(last, __shfl_xor(last, o, 64));
    count += __shfl_xor(count, o, 64);
  }
  first = uniform(first);
  end = uniform(count == last - first + 1 ? last + 1 : 0);
}

// ----------------------------------------------------------------------- host
inline int64_t dense_tiles(int64_t n) { return (n + 31) / 32; }

// k_dense.hip
park_status launch_doc_tiles(const DocIds& k, const DocIds* q, int B, hipStream_t st);
// tiles of 128 held rows against `tiles` streamed ones; uneven: the tiles'
// lengths differ (masks, sequences of their own)
DenseSplit dense_split(int64_t held, int64_t tiles, bool f32, bool uneven, bool causal, int per_cu,
                       int launch);
DenseSplit dense_fwd_split(int64_t rows, int64_t heads, int64_t key_tiles, int d, int dtype, bool cached,
                           bool uneven, bool causal);
park_status launch_dense_fwd(const DenseArgs& a, int d, int dtype, bool cached, hipStream_t st);

// what the backward kernels take beside the forward's arguments (q, k, v, o)
struct DenseGrad {
  RowsArg dout, dq, dk, dv;
  const float *lse, *dlse;  // [B][Hq][Nq] (dlse may be null)
  int o_f32;
  float* rows;              // [B Hkv][ceil(R / 32)][DENSE_RF][32] what the rows need
  const DocTile* q_tiles;   // [B][ceil(R / 32)] (with documents)
  DenseSplit ksplit;        // dK and dV: tiles of 128 keys, the rows in parts
  DenseSplit qsplit;        // dQ: tiles of 128 rows, the keys in parts
  float* part;              // sums of the split tiles' rows
};
// floats a packed row needs: -lse, D, last key, document, position in its tile,
// slope, the tile's first position, one unused
constexpr int DENSE_RF = 8;

// k_dense_bwd.hip
park_status launch_dense_bwd(const DenseArgs& a, const DenseGrad& g, int d, int dtype,
                             hipStream_t st);

// k_cache.hip
struct CacheAppend {
  RowsArg k, v;
  uint8_t *pk, *pv;
  int8_t *k_exp, *v_exp;
  const int *table, *lens, *n_new;
  int B, Hkv, N, d, dtype, page_shift, n_pages, max_pages;
  int* status;
};
park_status launch_cache_append(const CacheAppend& a, hipStream_t st);

}  // namespace park
