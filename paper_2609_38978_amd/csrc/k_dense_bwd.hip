// Gradients of the dense attention (k_dense.hip).  With P_ij = exp(x_ij - lse_i)
// and D_i = dO_i . O_i - dlse_i (= sum_j P_ij dO_i . v_j - dlse_i),
//   dV_j = sum_i P_ij dO_i,        dX_ij = P_ij (dO_i . v_j - D_i),
//   dS_ij = dX_ij (1 - tanh^2),    dQ_i = scale sum_j dS_ij k_j,
//   dK_j = scale sum_i dS_ij q_i   (over the rows of all heads that share j).
//
// Two kernels recompute the scores, one with query rows held and the keys
// streamed (dQ), one with keys held and the packed rows streamed (dK, dV), so
// that every sum has one owner and a fixed order: seven products instead of
// five, and no atomics.  P and dS are rounded to bf16 once, as operands of the
// products that sum them in float; with float inputs nothing is rounded.
//
// Bound by the matrix cores (8 heads of 16384 tokens, d = 128: dQ 1.4 ms =
// 1.16 PFLOP/s for its three products, dK and dV 1.9 ms = 1.14 for their four; the
// forward beside them 1.0 ms).  With documents of different lengths by their parts'
// uneven work and, with cap and bias, by vector instructions (2 x 16 heads of 4133
// rows in 5 documents: dQ 102 us, dK and dV 177, the CUs at work half of that).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dense.h"
#include "kernels.h"

namespace park {

// What the packed rows need, by tiles of 32 rows: field f of row r at
// rows[((b Hkv + hk) tiles + r / 32) DENSE_RF + f][r % 32].  Field 0 is the
// summand that turns a score into the exponent's argument (grad_exp: -lse times
// `unit`; -infinity for a row without keys, so that its probabilities are 0).
// Field 4 is the position less the tile's first, which field 6 has.
// Eight threads a row.
//
// Field 1 is D.  From an O that was rounded to bf16 it is off by 2^-9 of it or
// so, which the sums of dS spread over a row's keys; where there are few the
// difference dP - D is small and shows it (causal texts of 2 and 4 tokens: dQ and
// dK 0.01 and 0.0046 off in norm; 0.0032 and 0.0028 with D from its definition,
// sum_j P_ij dP_ij).  Rows that attend at most DENSE_NEAR keys take that if those
// are the first of all, or within DENSE_NEAR places of the row's own as those of a
// short document in a pack are.  It costs 14 us of the kernel's 51 for 64 x 24
// causal heads of 256 tokens, d = 128 (16 keys: 53, for 0.0025 instead of 0.0027 at
// 16 tokens), and of packs of 2 x 24 heads of 8192 tokens 12 us of 54, 18 of 60 and
// 55 of 97 where documents have 256, 32 and 4.
constexpr int DENSE_NEAR = 8;

// exp(x - lse) for a score x in the kernel's units, sl2 = log2(e) in them: one
// instruction beside the exponential with x0 = -lse log2(e); for float inputs the
// difference comes first (x0 = -lse in the scores' units), as in the forward
template <bool F32>
__device__ __forceinline__ float grad_exp(float x, float x0, float sl2) {
  return __builtin_amdgcn_exp2f(F32 ? (x + x0) * sl2 : fmaf(x, sl2, x0));
}

// elements part E .. part E + E - 1 of a row as they are stored
template <class T, int E>
struct RowPart {
  static constexpr int W = sizeof(T) == 4 ? E : E / 2;
  alignas(16) uint32_t w[W];
  __device__ __forceinline__ RowPart(const char* p, int part) {
    p += part * (E * (int)sizeof(T));
#pragma unroll
    for (int e = 0; e < W; e += 4) *(uint4*)(w + e) = *(const uint4*)(p + 4 * e);
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return bf2f((bf16_t)(w[e / 2] >> 16 * (e & 1)));
  }
};
template <int E, class A, class B>
__device__ __forceinline__ float dot_part(const A& a, const B& b) {
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) s = fmaf(a[e], b[e], s);
  return s;
}

// ... of two rows of one type: bf16 in pairs (the products exact, sums in float)
template <class T, int E>
__device__ __forceinline__ float dot_rows(const RowPart<T, E>& a, const RowPart<T, E>& b) {
  if constexpr (sizeof(T) == 4) return dot_part<E>(a, b);
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < E / 2; ++e)
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, a.w[e]),
                                        __builtin_bit_cast(bf16x2_t, b.w[e]), s, false);
  return s;
}

template <class T, class OT, int D>
__global__ __launch_bounds__(256) void k_dense_rows(const DenseArgs a, const DenseGrad g, float unit) {
  const int tiles = (a.R + 31) / 32, t = blockIdx.x % tiles, bh = blockIdx.x / tiles;
  const int b = bh / a.Hkv, hk = bh % a.Hkv, c = threadIdx.x >> 3, part = threadIdx.x & 7;
  const int r = t * 32 + c, qi = r / a.G, hq = hk * a.G + r % a.G;
  float* out = g.rows + (size_t)blockIdx.x * (DENSE_RF * 32) + c;
  float x0 = -INFINITY, dd = 0.0f, slope = 0.0f;
  int jlim = -1, doc = -1;
  const int pos = qi + a.q_pos;
  const size_t at = ((size_t)b * a.Hkv * a.G + hq) * a.Nq + qi;  // (r < R)
  // documents of the 17 keys around the row's own place, one or two a lane
  const int base = max(min(pos, a.Nk - 1) - DENSE_NEAR, 0);
  int id[3] = {-1, -1, -1};
  if (r < a.R) {
    const char* o = a.o.p + b * a.o.b + hq * a.o.h + qi * a.o.r;
    const char* dout = g.dout.p + b * g.dout.b + hq * g.dout.h + qi * g.dout.r;
    constexpr int E = D / 8;
    dd = dot_part<E>(RowPart<T, E>(dout, part), RowPart<OT, E>(o, part));
    const float lse = g.lse[at];
    x0 = lse == INFINITY ? NAN : -lse * unit;
    if (lse == -INFINITY) x0 = -INFINITY;
    jlim = a.Nk - 1;
    if (a.causal) jlim = min(jlim, max(pos, a.prefix ? a.prefix[b] - 1 : -1));
    if (a.q_doc) {
      doc = a.q_doc[(size_t)b * a.Nq + qi];
      if constexpr (sizeof(OT) == 2) {
        const int* ids = a.k_doc + (size_t)b * a.Nk;
#pragma unroll
        for (int i = 0; i < 3; ++i)  // (past the last: the last, which `ok` leaves out)
          id[i] = ids[min(base + DENSE_NEAR * i + (i < 2 ? part : 0), a.Nk - 1)];
      }
      if (doc < 0) jlim = -1;
    }
    if (a.slopes) slope = a.slopes[hq];
  }
  if constexpr (sizeof(OT) == 2) {
    // the keys of the row among the 17, as bits
    static_assert(DENSE_NEAR == 8, "eight lanes a row");
    uint32_t keys = jlim >= 0 && jlim < DENSE_NEAR ? (2u << jlim) - 1u : 0u;
    bool all = true;  // it has no others
    if (a.q_doc) {
      keys = 0u;
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const bool ok = id[i] == doc && base + DENSE_NEAR * i + (i < 2 ? part : 0) <= jlim;
        keys |= ((uint32_t)(__ballot(ok) >> (threadIdx.x & 56)) & (i < 2 ? 255u : 1u)) << (8 * i);
      }
      if (__builtin_popcount(keys) > DENSE_NEAR) keys = 0u;
      all = base == 0 && jlim <= 2 * DENSE_NEAR;
    }
    if (keys) {
      const float sl2 = (a.cap > 0.0f || a.slopes ? 1.0f : a.scale) * 1.4426950408889634f;
      const int j0 = a.q_doc ? base : 0;
      const char* kp = a.k.p + b * a.k.b + hk * a.k.h + j0 * a.k.r;
      const char* vp = a.v.p + b * a.v.b + hk * a.v.h + j0 * a.v.r;
      constexpr int E = D / 8;
      const RowPart<T, E> q(a.q.p + b * a.q.b + hq * a.q.h + qi * a.q.r, part);
      const RowPart<T, E> y(g.dout.p + b * g.dout.b + hq * g.dout.h + qi * g.dout.r, part);
      float near = 0.0f, psum = 0.0f;
#pragma unroll 1  // (few rows come here: registers for the others' loads)
      for (; keys; keys &= keys - 1) {
        const int i = __builtin_ctz(keys);
        const RowPart<T, E> k(kp + i * a.k.r, part), v(vp + i * a.v.r, part);
        float x = dot_rows(q, k);
        const float dp = dot_rows(y, v);
#pragma unroll
        for (int s = 4; s > 0; s >>= 1) x += __shfl_xor(x, s, 8);
        if (a.cap > 0.0f) x = a.cap * dense_tanh(x, a);
        else if (a.slopes) x *= a.scale;
        x = fmaf(-slope, (float)abs(pos - j0 - i), x);
        const float p = grad_exp<sizeof(T) == 4>(x, x0, sl2);
        psum += p;
        near = fmaf(p, dp, near);
      }
      // (elsewhere it may have others: what those weigh is what these lack)
      if (all || psum > 1.0f - 0x1p-11f) dd = near;
    }
  }
  if (g.dlse && part == 0 && r < a.R) dd -= g.dlse[at];
#pragma unroll
  for (int s = 4; s > 0; s >>= 1) dd += __shfl_xor(dd, s, 8);
  const int first = 32 * t / a.G + a.q_pos;
  const float f[DENSE_RF] = {x0, dd, __int_as_float(jlim), __int_as_float(doc),
                             (float)(pos - first), slope, __int_as_float(first), 0.0f};
  static_assert(DENSE_RF == 8, "a field per thread");
#pragma unroll
  for (int k = 0; k < DENSE_RF; ++k)
    if (part == k) out[32 * k] = f[k];
}

// 16-byte copies to LDS from addresses of their own
__device__ __forceinline__ void lds_dma16_far(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(lds)
               : "memory", "m0");
}

// Score variants on a tile: st becomes the scores in their final units (raw
// products without variants) and gate the tanh's derivative.  far(q): distance
// of register q's pair; slope(q) its head's slope.
template <class Far, class Slope>
__device__ __forceinline__ void grad_variants(const DenseArgs& a, f32x16_t& st, f32x16_t& gate,
                                              Far far, Slope slope) {
  if (a.cap > 0.0f) {
    dense_cap_tile<true>(st, a, &gate);
  } else {
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      st[q] *= a.scale;
      gate[q] = 1.0f;
    }
  }
  if (a.slopes) {
#pragma unroll
    for (int q = 0; q < 16; ++q) st[q] = fmaf(-slope(q), fabsf(far(q)), st[q]);
  }
}

// dQ: 128 packed rows held, keys and values streamed
template <class T, int D, bool MOD>
__global__ __launch_bounds__(256, (sizeof(T) == 4 && D == 128) ? 1
                                  : sizeof(T) * D == 128       ? 3
                                                               : 2) void k_dense_dq(const DenseArgs a,
                                                                                    const DenseGrad g) {
  using TL = DenseTile<T, D>;
  using frag = typename DenseOp<T>::frag;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int KS = D / 16, DB = D / 32, NS = 2, ES = sizeof(T);
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  unsigned char *kt = smem, *vt = smem + NS * TL::BYTES;
  __shared__ int red[8];
  __shared__ __attribute__((aligned(16))) int kds[NS][64];  // documents of a tile's keys
  const int tid = threadIdx.x, w = uniform(tid >> 6);
  const int l = tid & 63, hf = l >> 5, c32 = l & 31;
  const int nrt = (a.R + DENSE_ROWS - 1) / DENSE_ROWS;
  const DenseItem it = dense_item(g.qsplit, a.B * a.Hkv, nrt, a.causal, true, blockIdx.x);
  const int rt = it.tile, bh = it.head;
  const int b = uniform(bh / a.Hkv), hk = uniform(bh % a.Hkv);
  const int r = rt * DENSE_ROWS + 32 * w + c32;
  const int qi = r / a.G, hq = hk * a.G + r % a.G;
  const bool exists = r < a.R;
  // (a row of no document needs no mask: its gradient is 0 in the end)
  bool valid = exists;
  float x0 = -INFINITY, dd = 0.0f, slope = 0.0f;
  int jlim = a.Nk - 1, qd = 0;
  const int pos = qi + a.q_pos;
  if (exists) {
    const float* f = g.rows + ((size_t)bh * ((a.R + 31) / 32) + (r >> 5)) * (DENSE_RF * 32) + (r & 31);
    x0 = f[0];
    dd = f[32];
    jlim = __float_as_int(f[64]);
    qd = __float_as_int(f[96]);
    slope = f[160];
  }
  const bool docs = a.q_doc != nullptr;
  if (docs && exists && qd < 0) {
    valid = false;
    jlim = a.Nk - 1;
  }
  int jtop = valid ? jlim : -1, jfull = jlim;
  int qlo = valid && qd >= 0 ? qd : 0x7fffffff, qhi = valid ? qd : -1;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    jtop = max(jtop, __shfl_xor(jtop, o, 64));
    jfull = min(jfull, __shfl_xor(jfull, o, 64));
    qlo = min(qlo, __shfl_xor(qlo, o, 64));
    qhi = max(qhi, __shfl_xor(qhi, o, 64));
  }
  jtop = uniform(jtop);
  jfull = uniform(jfull);
  qlo = uniform(qlo);
  qhi = uniform(qhi);
  int none = 0, jend = jtop;
  wg_range<4>(none, jend, red);
  int tbeg = 0, tend = (jend + 32) >> 5;
  const DocTile* kd = a.k_tiles + (size_t)b * ((a.Nk + 31) / 32);
  if (docs && tend > 0) {
    int lo = qlo, hi = qhi, first, last;
    wg_range<4>(lo, hi, red);
    doc_range<4>(kd, tend, lo, hi, red, first, last);
    tbeg = first;
    tend = last + 1;
  }
  if (it.part >= 0) dense_part(it.part, g.qsplit.n, tbeg, tend);
  tbeg = uniform(tbeg);
  tend = uniform(tend);
  frag qf[KS], df[KS];
  {
    const char* qp = a.q.p + b * a.q.b + hq * a.q.h + qi * a.q.r + 8 * hf * ES;
    const char* dp = g.dout.p + b * g.dout.b + hq * g.dout.h + qi * g.dout.r + 8 * hf * ES;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[s] = frag{};
      df[s] = frag{};
      if (valid) {
        dense_load(qf[s], qp + 16 * s * ES);
        dense_load(df[s], dp + 16 * s * ES);
      }
    }
  }
  const float sl2 = MOD ? 1.4426950408889634f : a.scale * 1.4426950408889634f;
  const char* kp = a.k.p + b * a.k.b + hk * a.k.h;
  const char* vp = a.v.p + b * a.v.b + hk * a.v.h;
  const uint32_t lk = (uint32_t)((l >> 2) * a.k.r) + TL::copy_byte(0, l);
  const uint32_t lv = (uint32_t)((l >> 2) * a.v.r) + TL::copy_byte(0, l);
  auto issue = [&](int t, int sl) {
#pragma unroll
    for (int i = 0; i < TL::NI; ++i) {
      const int c = w * TL::NI + i;
      const uint32_t dk = lds_addr(kt) + sl * TL::BYTES + 1024 * c;
      const uint32_t dv = lds_addr(vt) + sl * TL::BYTES + 1024 * c;
      const char *ks = kp + (int64_t)t * 32 * a.k.r, *vs = vp + (int64_t)t * 32 * a.v.r;
      if (32 * t + 32 <= a.Nk) {
        lds_dma16(ks + 16 * (c & 1) * a.k.r + 64 * (c >> 1), lk, dk);
        lds_dma16(vs + 16 * (c & 1) * a.v.r + 64 * (c >> 1), lv, dv);
      } else {  // rows past the last: the last
        const int64_t row = min(TL::copy_row(c, l), a.Nk - 1 - 32 * t);
        lds_dma16(ks, (uint32_t)(row * a.k.r) + TL::copy_byte(c, l), dk);
        lds_dma16(vs, (uint32_t)(row * a.v.r) + TL::copy_byte(c, l), dv);
      }
    }
    // (the same from every wavefront; rows past the last: the last)
    if (docs)
      lds_dma4(a.k_doc + (size_t)b * a.Nk, 4 * (uint32_t)min(32 * t + l, a.Nk - 1), lds_addr(kds[sl]));
  };
  static_assert(TL::DW == 4, "every wavefront copies");
  f32x16_t acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x16_t{};
  // Tiles [mlo, mhi) are allowed whole for every row of the wavefront.
  int mlo = tbeg, mhi = min((jfull + 1) >> 5, tend);
  if (docs) {
    int end;
    doc_run(kd, tbeg, tend, qlo == qhi ? qlo : -1, mlo, end);
    mhi = min(mhi, end);
  }
  if (tbeg < tend) issue(tbeg, 0);
  // one barrier a tile: tile t has landed and the slot of tile t - 1 is read
  auto arrive = [&](int t) {
    wait_vmcnt<0>();
    __syncthreads();
    if (t + 1 < tend) issue(t + 1, (t + 1 - tbeg) & 1);
  };
  auto tile = [&](auto masked, int t) {
    const int sl = (t - tbeg) & 1;
    const uint32_t ks = lds_addr(kt) + sl * TL::BYTES + TL::row_at(l);
    const uint32_t vs = lds_addr(vt) + sl * TL::BYTES + TL::row_at(l);
    const uint32_t kc = lds_addr(kt) + sl * TL::BYTES + TL::col_at(l);
    f32x16_t st = {}, dp = {}, gate;
    // (the score products first: 2 % of the whole gradient, 4.72 -> 4.63 ms of a
    // step of 8 x 16384 tokens; in the forward it costs 5 %)
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      st = dense_mma(dense_row_raw<T, D>(ks, s), qf[s], st);
      dp = dense_mma(dense_row_raw<T, D>(vs, s), df[s], dp);
    }
    __builtin_amdgcn_s_setprio(0);
    const float far0 = (float)(pos - 32 * t - 4 * hf);
    if constexpr (MOD)
      grad_variants(a, st, gate, [&](int q) { return far0 - (float)(8 * (q >> 2) + (q & 3)); },
                    [&](int) { return slope; });
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const float p = grad_exp<F32>(st[q], x0, sl2);
      st[q] = p * (dp[q] - dd);
      if constexpr (MOD) st[q] *= gate[q];
    }
    if constexpr (masked.value) {
      const int j0 = opaque(32 * t + 4 * hf);
      const int* kdoc = &kds[sl][4 * hf];
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        uint32_t ok = bit_ge0(jlim - j0 - 8 * (q >> 2) - (q & 3));
        if (docs) ok &= 1u - bit_ne0(kdoc[8 * (q >> 2) + (q & 3)] ^ qd);
        st[q] = mask_zero(st[q], ok, 0);
      }
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      frag sf;
      dense_pack(sf, st, kk);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        frag f = dense_col_raw<T, D>(kc, kk, db);
        // a key that is not finite has reached the scores of the rows that
        // allow it; the others have nothing of it
        if constexpr (masked.value) dense_fix(f);
        acc[db] = dense_mma(f, sf, acc[db]);
      }
    }
  };
  int t = tbeg;
  while (t < tend) {
    if (!F32 && t >= mlo && t < mhi) {
      for (; t < mhi; ++t) {  // (most tiles: no masking in the loop)
        arrive(t);
        tile(std::bool_constant<F32>{}, t);
      }
    } else {
      arrive(t);
      if (32 * t <= jtop) tile(std::true_type{}, t);
      ++t;
    }
  }
  if (!exists) return;
  if (!valid) {
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = f32x16_t{};
  }
  if (it.part >= 0) {
    float* o = g.part + ((size_t)it.slot * DENSE_ROWS + 32 * w + c32) * D + 4 * hf;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q = 0; q < 16; q += 4)
        *(float4*)(o + 32 * db + 2 * q) =
            make_float4(acc[db][q], acc[db][q + 1], acc[db][q + 2], acc[db][q + 3]);
    return;
  }
  char* o = g.dq.p + b * g.dq.b + hq * g.dq.h + qi * g.dq.r;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int q = 0; q < 16; q += 4)
      store_out4<T>((T*)o + 32 * db + 2 * q + 4 * hf, acc[db][q] * a.scale, acc[db][q + 1] * a.scale,
                    acc[db][q + 2] * a.scale, acc[db][q + 3] * a.scale);
}

// dK, dV: 128 keys held, the packed rows' queries and output gradients streamed
//
// At d = 128 the sums (128 registers) leave no room for keys and values beside
// them at two wavefronts a SIMD: the values stay in LDS.
template <class T, int D, bool MOD>
__global__ __launch_bounds__(256, (sizeof(T) == 2 ? 2 : 1)) void k_dense_dkv(const DenseArgs a,
                                                                            const DenseGrad g) {
  using TL = DenseTile<T, D>;
  using frag = typename DenseOp<T>::frag;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int KS = D / 16, DB = D / 32, NS = 2, ES = sizeof(T), RB = DENSE_RF * 32 * 4;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  constexpr bool VL = D == 128;  // values in LDS
  unsigned char *qt = smem, *ot = smem + NS * TL::BYTES, *rt = smem + 2 * NS * TL::BYTES;
  unsigned char* vt = rt + 2 * RB;  // (VL) [4] value tiles
  __shared__ int red[8];
  const int tid = threadIdx.x, w = uniform(tid >> 6);
  const int l = tid & 63, hf = l >> 5, c32 = l & 31;
  const int nkt = (a.Nk + DENSE_ROWS - 1) / DENSE_ROWS;
  const DenseItem it = dense_item(g.ksplit, a.B * a.Hkv, nkt, a.causal, false, blockIdx.x);
  const int kt = it.tile, bh = it.head;
  const int b = uniform(bh / a.Hkv), hk = uniform(bh % a.Hkv);
  const int j0 = kt * DENSE_ROWS, jw = j0 + 32 * w, j = jw + c32;
  const bool valid = j < a.Nk;
  const bool docs = a.q_doc != nullptr;
  const int kdoc = docs && valid ? a.k_doc[(size_t)b * a.Nk + j] : -1;
  int klo = kdoc >= 0 ? kdoc : 0x7fffffff, khi = kdoc;
  const int pre = a.prefix ? a.prefix[b] : 0;
  const int tiles = (a.R + 31) / 32;
  int tbeg = 0, tend = tiles;
  if (a.causal && j0 >= pre) {
    const int64_t i0 = max((int64_t)j0 - a.q_pos, (int64_t)0);  // first query that sees a key
    tbeg = (int)min((int64_t)tiles, (i0 * a.G) >> 5);
  }
  if (docs) {
    int lo = klo, hi = khi, first, last;
    wg_range<4>(lo, hi, red);
    doc_range<4>(g.q_tiles + (size_t)b * tiles, tiles, lo, hi, red, first, last);
    tbeg = max(tbeg, first);
    tend = last + 1;
  }
  if (it.part >= 0) dense_part(it.part, g.ksplit.n, tbeg, tend);
  tbeg = uniform(tbeg);
  tend = uniform(tend);
  // ids of the wavefront's keys (for tiles of one document)
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    klo = min(klo, __shfl_xor(klo, o, 64));
    khi = max(khi, __shfl_xor(khi, o, 64));
  }
  klo = uniform(klo);
  khi = uniform(khi);
  // Tiles [mlo, mhi) are allowed whole for the wavefront's keys; before `tsee`
  // no row sees one of them.
  int mlo = tbeg, mhi = min(a.R >> 5, tend), tsee = jw < a.Nk ? tbeg : tend;
  if (a.causal) {
    auto tile_of = [&](int key, bool up) {  // tile of the first row whose query is at `key` or past it
      const int64_t r = max((int64_t)key - a.q_pos, (int64_t)0) * a.G;
      return (int)min((up ? r + 31 : r) >> 5, (int64_t)tend);
    };
    if (jw + 31 >= pre) mlo = max(mlo, tile_of(jw + 31, true));
    if (jw >= pre) tsee = max(tsee, tile_of(jw, false));
  }
  if (docs) {
    int first, end;
    doc_run(g.q_tiles + (size_t)b * tiles, tbeg, tend,
            klo == khi ? klo : -1, first, end);
    mlo = max(mlo, first);
    mhi = min(mhi, end);
  }
  frag kf[KS], vf[VL ? 1 : KS];
  {
    const char* kp = a.k.p + b * a.k.b + hk * a.k.h + j * a.k.r + 8 * hf * ES;
    const char* vp = a.v.p + b * a.v.b + hk * a.v.h;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      kf[s] = frag{};
      if (valid) dense_load(kf[s], kp + 16 * s * ES);
      if constexpr (!VL) {
        vf[s] = frag{};
        if (valid) dense_load(vf[s], vp + j * a.v.r + 8 * hf * ES + 16 * s * ES);
      }
    }
    if constexpr (VL) {
      // this wavefront's 32 values (past the last: the last, in lanes nobody reads)
#pragma unroll
      for (int c = 0; c < TL::NDMA; ++c) {
        lds_dma16_far(vp + min(jw + TL::copy_row(c, l), a.Nk - 1) * a.v.r + TL::copy_byte(c, l),
                      lds_addr(vt) + w * TL::BYTES + 1024 * c);
      }
    }
  }
  auto v_frag = [&](int s) {
    if constexpr (VL) return dense_row_raw<T, D>(lds_addr(vt) + w * TL::BYTES + TL::row_at(l), s);
    else return vf[s];
  };
  const float sl2 = MOD ? 1.4426950408889634f : a.scale * 1.4426950408889634f;
  const char* qp = a.q.p + b * a.q.b + (int64_t)hk * a.G * a.q.h;
  const char* dp = g.dout.p + b * g.dout.b + (int64_t)hk * a.G * g.dout.h;
  auto issue = [&](int t, int sl) {
#pragma unroll
    for (int i = 0; i < TL::NI; ++i) {
      const int c = w * TL::NI + i;
      const uint32_t lq = lds_addr(qt) + sl * TL::BYTES + 1024 * c;
      const uint32_t lo = lds_addr(ot) + sl * TL::BYTES + 1024 * c;
      if (a.G == 1 && 32 * t + 32 <= a.R) {
        const uint32_t at = TL::copy_byte(0, l);
        lds_dma16(qp + (32 * (int64_t)t + 16 * (c & 1)) * a.q.r + 64 * (c >> 1),
                  (uint32_t)((l >> 2) * a.q.r) + at, lq);
        lds_dma16(dp + (32 * (int64_t)t + 16 * (c & 1)) * g.dout.r + 64 * (c >> 1),
                  (uint32_t)((l >> 2) * g.dout.r) + at, lo);
      } else {
        const int r = min(t * 32 + TL::copy_row(c, l), a.R - 1);
        const int qi = a.G == 1 ? r : (int)(__umulhi((uint32_t)r, a.gmul) >> (a.gshift - 1));
        const int gq = r - qi * a.G;
        lds_dma16_far(qp + qi * a.q.r + gq * a.q.h + TL::copy_byte(c, l), lq);
        lds_dma16_far(dp + qi * g.dout.r + gq * g.dout.h + TL::copy_byte(c, l), lo);
      }
    }
    // the rows' fields: 256 bytes a wavefront
    lds_dma4((const char*)g.rows + ((size_t)bh * tiles + t) * RB, 256 * w + 4 * l,
             lds_addr(rt) + sl * RB + 256 * w);
  };
  static_assert(TL::DW == 4 && RB == 4 * 256, "every wavefront copies");
  f32x16_t dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    dk[db] = f32x16_t{};
    dv[db] = f32x16_t{};
  }
  if (tbeg < tend) issue(tbeg, 0);
  auto arrive = [&](int t) {  // as for dQ
    wait_vmcnt<0>();
    __syncthreads();
    if (t + 1 < tend) issue(t + 1, (t + 1 - tbeg) & 1);
  };
  auto tile = [&](auto masked, int t) {
    const int sl = (t - tbeg) & 1;
    const uint32_t qs = lds_addr(qt) + sl * TL::BYTES + TL::row_at(l);
    const uint32_t os = lds_addr(ot) + sl * TL::BYTES + TL::row_at(l);
    const uint32_t qc = lds_addr(qt) + sl * TL::BYTES + TL::col_at(l);
    const uint32_t oc = lds_addr(ot) + sl * TL::BYTES + TL::col_at(l);
    const float* rf = (const float*)(rt + sl * RB) + 4 * hf;  // row 8 b + r of this half
    auto field = [&](int f, int q) { return rf[32 * f + 8 * (q >> 2) + (q & 3)]; };
    f32x16_t st = {}, ds = {}, gate;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      st = dense_mma(dense_row_raw<T, D>(qs, s), kf[s], st);
      ds = dense_mma(dense_row_raw<T, D>(os, s), v_frag(s), ds);
    }
    __builtin_amdgcn_s_setprio(0);
    if constexpr (MOD) {
      const float far0 = (float)(__float_as_int(field(6, 0)) - j);
      grad_variants(a, st, gate, [&](int q) { return far0 + field(4, q); },
                    [&](int q) { return field(5, q); });
    }
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      st[q] = grad_exp<F32>(st[q], field(0, q), sl2);
      ds[q] = st[q] * (ds[q] - field(1, q));
      if constexpr (MOD) ds[q] *= gate[q];
    }
    uint32_t bits = 0u;
    if constexpr (masked.value) {
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const uint32_t ok = bit_ge0(__float_as_int(field(2, q)) - j);
        bits |= (docs ? ok & (1u - bit_ne0(__float_as_int(field(3, q)) ^ kdoc)) : ok) << q;
      }
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        st[q] = mask_zero(st[q], bits, q);
        ds[q] = mask_zero(ds[q], bits, q);
      }
    }
    frag pf[2], sf[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      dense_pack(pf[kk], st, kk);
      dense_pack(sf[kk], ds, kk);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      frag f[2], y[2];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        f[kk] = dense_col_raw<T, D>(oc, kk, db);
        y[kk] = dense_col_raw<T, D>(qc, kk, db);
        if constexpr (masked.value) dense_fix(y[kk]);  // (it has reached its scores)
      }
      if constexpr (masked.value) dense_guard(f, valid ? bits : 0u, dv[db]);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        dv[db] = dense_mma(f[kk], pf[kk], dv[db]);
        dk[db] = dense_mma(y[kk], sf[kk], dk[db]);
      }
    }
  };
  int t = tbeg;
  while (t < tend) {
    if (!F32 && t >= mlo && t < mhi) {
      for (; t < mhi; ++t) {  // (most tiles: no masking in the loop)
        arrive(t);
        tile(std::bool_constant<F32>{}, t);
      }
    } else {
      arrive(t);
      if (t >= tsee) tile(std::true_type{}, t);
      ++t;
    }
  }
  if (!valid) return;
  if (docs && kdoc < 0) {  // (a key of no document asked for no mask)
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      dk[db] = f32x16_t{};
      dv[db] = f32x16_t{};
    }
  }
  if (it.part >= 0) {
    float* ok = g.part + ((size_t)it.slot * DENSE_ROWS + 32 * w + c32) * D + 4 * hf;
    float* ov = ok + g.ksplit.rows(DENSE_ROWS) * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q = 0; q < 16; q += 4) {
        *(float4*)(ok + 32 * db + 2 * q) =
            make_float4(dk[db][q], dk[db][q + 1], dk[db][q + 2], dk[db][q + 3]);
        *(float4*)(ov + 32 * db + 2 * q) =
            make_float4(dv[db][q], dv[db][q + 1], dv[db][q + 2], dv[db][q + 3]);
      }
    return;
  }
  char* ok = g.dk.p + b * g.dk.b + hk * g.dk.h + j * g.dk.r;
  char* ov = g.dv.p + b * g.dv.b + hk * g.dv.h + j * g.dv.r;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int q = 0; q < 16; q += 4) {
      const int c = 32 * db + 2 * q + 4 * hf;
      store_out4<T>((T*)ok + c, dk[db][q] * a.scale, dk[db][q + 1] * a.scale,
                    dk[db][q + 2] * a.scale, dk[db][q + 3] * a.scale);
      store_out4<T>((T*)ov + c, dv[db][q], dv[db][q + 1], dv[db][q + 2], dv[db][q + 3]);
    }
}

// out = f sum_s part[s], in the parts' order, for the rows of the split tiles;
// heads of N G packed rows, four columns a thread
template <class T, int D>
__global__ __launch_bounds__(256) void k_dense_sum(const float* __restrict__ part, DenseSplit sp,
                                                   RowsArg o, RowsArg o2, int B, int Hkv, int G,
                                                   int rows, int causal, int last_first, float f) {
  if (blockIdx.y) {  // (dV beside dK)
    part += sp.rows(DENSE_ROWS) * D;
    o = o2;
    f = 1.0f;
  }
  const int at = blockIdx.x * (1024 / D) + threadIdx.x / (D / 4), c = threadIdx.x % (D / 4) * 4;
  const int tiles = (rows + DENSE_ROWS - 1) / DENSE_ROWS, heads = B * Hkv;
  const int unit = sp.whole + at / DENSE_ROWS;  // (as dense_item has them)
  const int bh = causal ? unit % heads : unit / tiles, t = causal ? unit / heads : unit % tiles;
  const int r = (last_first ? tiles - 1 - t : t) * DENSE_ROWS + at % DENSE_ROWS;
  if (at >= sp.rest * DENSE_ROWS || r >= rows) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < sp.n; ++i) {
    const float4 x = *(const float4*)(part + ((size_t)i * sp.rest * DENSE_ROWS + at) * D + c);
    s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
  }
  const int b = bh / Hkv;
  char* p = o.p + b * o.b + (int64_t)(bh % Hkv * G + r % G) * o.h + r / G * o.r;
  store_out4<T>((T*)p + c, s.x * f, s.y * f, s.z * f, s.w * f);
}

template <class T, int D, bool MOD>
static park_status bwd_launch(const DenseArgs& a, const DenseGrad& g, hipStream_t st) {
  using TL = DenseTile<T, D>;
  constexpr size_t ldq = 4 * TL::BYTES,
                   ldk = 4 * TL::BYTES + 2 * DENSE_RF * 32 * 4 + (D == 128 ? 4 * TL::BYTES : 0);
  static std::atomic<uint64_t> dq_done{0}, dk_done{0};
  PARK_TRY(reserve_lds((const void*)k_dense_dq<T, D, MOD>, ldq, dq_done, "attention gradient"));
  PARK_TRY(reserve_lds((const void*)k_dense_dkv<T, D, MOD>, ldk, dk_done, "attention gradient"));
  const int64_t heads = (int64_t)a.B * a.Hkv;
  if (a.R > 0) {
    const dim3 grid((unsigned)(heads * dense_tiles(a.R)));
    const float unit = sizeof(T) == 2 ? 1.4426950408889634f : MOD ? 1.0f : 1.0f / a.scale;
    if (g.o_f32)
      PARK_LAUNCH("dense_rows", (k_dense_rows<T, float, D>), grid, dim3(256), 0, st, a, g, unit);
    else
      PARK_LAUNCH("dense_rows", (k_dense_rows<T, bf16_t, D>), grid, dim3(256), 0, st, a, g, unit);
  }
  auto sums = [&](const DenseSplit& sp, const RowsArg& o, const RowsArg* o2, int G, int rows,
                  int last) -> park_status {
    PARK_LAUNCH("dense_sum", (k_dense_sum<T, D>),
                dim3(sp.rest * DENSE_ROWS / (1024 / D), o2 ? 2 : 1), dim3(256), 0, st,
                (const float*)g.part, sp, o, o2 ? *o2 : o, a.B, a.Hkv, G, rows, a.causal, last, a.scale);
    return PARK_OK;
  };
  if (a.Nk > 0) {
    PARK_LAUNCH("dense_dkv", (k_dense_dkv<T, D, MOD>), dim3((unsigned)g.ksplit.groups()), dim3(256),
                ldk, st, a, g);
    if (g.ksplit.rest) PARK_TRY(sums(g.ksplit, g.dk, &g.dv, 1, a.Nk, 0));
  }
  if (a.R > 0) {
    PARK_LAUNCH("dense_dq", (k_dense_dq<T, D, MOD>), dim3((unsigned)g.qsplit.groups()), dim3(256), ldq,
                st, a, g);
    if (g.qsplit.rest) PARK_TRY(sums(g.qsplit, g.dq, nullptr, a.G, a.R, 1));
  }
  return PARK_OK;
}

template <class T>
static park_status bwd_type(const DenseArgs& a, const DenseGrad& g, int d, hipStream_t st) {
  const bool mod = a.cap > 0.0f || a.slopes;
  if (d == 128) return mod ? bwd_launch<T, 128, true>(a, g, st) : bwd_launch<T, 128, false>(a, g, st);
  return mod ? bwd_launch<T, 64, true>(a, g, st) : bwd_launch<T, 64, false>(a, g, st);
}

park_status launch_dense_bwd(const DenseArgs& a, const DenseGrad& g, int d, int dtype,
                             hipStream_t st) {
  return dtype == PARK_BF16 ? bwd_type<bf16_t>(a, g, d, st) : bwd_type<float>(a, g, d, st);
}

}  // namespace park
