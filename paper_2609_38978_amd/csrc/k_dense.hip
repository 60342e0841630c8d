// Dense attention forward: O_i = softmax_j(x_ij) v_j over the keys a mask
// allows, with capped scores and a distance bias, on given keys (bf16, float)
// or on the pages of an 8-bit cache; lse_i = log sum_j exp x_ij.
//
// One pass over the keys with a running maximum and sum per query (the softmax
// is invariant to the shift).  A workgroup holds 128 packed query rows, 32 per
// wavefront, in registers and streams tiles of 32 keys and values through LDS.
// S^T = K Q^T leaves a query's scores in one lane pair, so that the row's maximum
// and sum take one exchange and the probabilities, rounded to bf16, are the
// operand of O^T = V^T P^T without leaving the registers.
//
// Work: 4 d per allowed pair, on the matrix cores; Q, O once, K and V once for
// every 128 packed rows (from L2: tiles of one head run side by side).
//   long keys: bound by the matrix cores and, beside them, by 16 exponentials a
//     tile and lane: 24 heads of 32400 tokens, d = 128, 11.8 ms = 1.10 PFLOP/s
//     (a library product of 16384 reaches 1.37 on the same card)
//   float: by the float MFMA, 1/16 of the bf16 rate: 4096 rows, d = 64, cap,
//     63.6 us = 68 TFLOP/s of 152
//   few keys (257 of 24 x 2 heads of 8449 rows): by reading Q and writing O and
//     by the latency of a workgroup's start: 90 us = 2.4 TB/s of 4.86
//   single tokens on the cache: by reading it: 32 sequences of 700..16384 tokens,
//     8 heads, 132 us = 4.2 TB/s
//   many queries on 64-wide pages with a cap: by vector instructions (e4m3 to
//     bf16 in every wavefront, the cap; the units are busy 0.59 of the cycles):
//     198 us = 0.30 PFLOP/s
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dense.h"
#include "kernels.h"

namespace park {

// document ids of 32-row tiles, of the keys or (a gradient's call) of both sides
__global__ __launch_bounds__(256) void k_doc_tiles(const DocIds k, const DocIds q, int B) {
  const DocIds& d = blockIdx.y ? q : k;
  const int tiles = d.tiles(), per = (tiles + 7) / 8, b = blockIdx.x / per;
  const int t = (blockIdx.x - b * per) * 8 + (threadIdx.x >> 5), l = threadIdx.x & 31;
  if (b >= B || t >= tiles) return;
  const int r = t * 32 + l, id = r < d.N * d.G ? d.ids[(size_t)b * d.N + r / d.G] : -1;
  int lo = id >= 0 ? id : 0x7fffffff, hi = id, least = id;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor(lo, o, 32));
    hi = max(hi, __shfl_xor(hi, o, 32));
    least = min(least, __shfl_xor(least, o, 32));
  }
  if (l == 0) d.out[(size_t)b * tiles + t] = {lo, hi, least >= 0 && lo == hi, 0};
}

park_status launch_doc_tiles(const DocIds& k, const DocIds* q, int B, hipStream_t st) {
  const int most = std::max(k.tiles(), q ? q->tiles() : 0);
  PARK_LAUNCH("doc_tiles", k_doc_tiles, dim3((unsigned)B * ((most + 7) / 8), q ? 2 : 1), dim3(256), 0,
              st, k, q ? *q : k, B);
  return PARK_OK;
}

// LDS of one ring of key and value tiles
template <class T, int D>
constexpr size_t dense_ring() {
  return 8 * (size_t)DenseTile<T, D>::BYTES;
}
// wavefronts of the form for few rows: as many rings as 128 KB hold
template <class T, int D>
constexpr int dense_few_waves() {
  return 4 * dense_ring<T, D>() <= 131072 ? 4 : 2 * dense_ring<T, D>() <= 131072 ? 2 : 1;
}

// T: type of the keys and values (fp8_t: pages of a cache, bf16 queries).
// FEW: at most 32 rows a head (single tokens).  The wavefronts of a workgroup
// then hold the same rows, take the keys in parts of their own through rings of
// their own, without barriers, and join at the end: reading the keys is what
// bounds it, and four times the copies are in flight.
// Workgroups a CU: two for the registers of a tile; three (168 registers) for
// pages of 64 values, whose conversion keeps the vector units busy (1500 queries
// over 3000..9001 keys, 16 heads, cap: 278 us with two, 242 with three and 206
// cut for them; keys in bf16 lose by it, 390 -> 396 us of a gradient's call).
template <class T, int D, bool MOD, bool FEW>
__global__ __launch_bounds__((FEW ? 64 * dense_few_waves<T, D>() : 256),
                             (FEW || (sizeof(T) == 4 && D == 128)) ? 1
                             : sizeof(T) * D == 64                 ? 3
                                                                   : 2) void k_dense_fwd(const DenseArgs a) {
  using TL = DenseTile<T, D>;
  using frag = typename DenseOp<T>::frag;
  constexpr bool F8 = sizeof(T) == 1, F32 = sizeof(T) == 4;
  constexpr int QS = F32 ? 4 : 2;  // bytes of a query element
  constexpr int KS = D / 16, DB = D / 32, NS = 4;  // ring slots, of keys and of values
  // tiles between the one whose scores are being turned into probabilities and
  // the one whose keys are read from LDS (float reads them at their use)
  constexpr int KA = F32 ? 1 : 2;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  constexpr int NW = FEW ? dense_few_waves<T, D>() : 4, ROWS = FEW ? 32 : DENSE_ROWS;
  constexpr int NI = FEW ? TL::NDMA : TL::NI;  // copies of a wavefront per tensor and tile
  static_assert(2 * NS * (size_t)TL::BYTES == dense_ring<T, D>(), "ring size");
  const int tid = threadIdx.x, w = uniform(tid >> 6);
  const int l = tid & 63, hf = l >> 5, c32 = l & 31;
  uint32_t kt = lds_addr(smem);  // [NS] key tiles, then [NS] value tiles
  asm volatile("" : "+s"(kt));   // (a number, not the address of an object)
  if constexpr (FEW) kt += w * (uint32_t)dense_ring<T, D>();
  const uint32_t vt = kt + NS * TL::BYTES;
  constexpr uint32_t RING = NS * TL::BYTES;
  // (F8) page id or -1, its two exponents
  int2* ptab = (int2*)(smem + (FEW ? NW : 1) * dense_ring<T, D>());
  __shared__ int red[3 * NW], bad_pages;
  // documents of the keys of pairs of tiles (four pairs)
  __shared__ __attribute__((aligned(16))) int kds[FEW ? 1 : 4][64];

  const int nrt = (a.R + ROWS - 1) / ROWS;
  const DenseItem it = dense_item(a.split, a.B * a.Hkv, nrt, a.causal, true, blockIdx.x);
  const int rt = it.tile, bh = it.head;
  const int b = uniform(bh / a.Hkv), hk = uniform(bh % a.Hkv);

  // this lane's packed row
  const int r = rt * ROWS + (FEW ? 0 : 32 * w) + c32;
  const int qi = r / a.G, hq = hk * a.G + r % a.G;
  int n = a.Nk, p0 = a.q_pos, nq = a.Nq;
  if constexpr (F8) {
    // (the queries end with the sequence; its keys, where the table does)
    const int len = max(a.lens[b], 0);
    n = min(len, a.max_pages << a.page_shift);
    if (a.q_lens) nq = min(max(a.q_lens[b], 0), a.Nq);
    p0 = len - nq;
    if (len > n && nq > 0 && a.status && tid == 0 && rt == 0 && hk == 0 && it.part <= 0)
      atomicOr(a.status, ST_BAD_PAGE);
  }
  const bool exists = r < a.R && qi < nq;
  bool valid = exists;
  // queries: the B operand of S^T = K Q^T
  frag qf[KS];
  {
    const char* qp = a.q.p + b * a.q.b + hq * a.q.h + qi * a.q.r + 8 * hf * QS;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[s] = frag{};
      if (exists) dense_load(qf[s], qp + 16 * s * QS);
    }
  }
  // the documents of the first 64 key tiles, one a lane
  const bool docs = a.q_doc != nullptr;
  const int ktiles = (a.Nk + 31) >> 5;
  const bool in_lanes = docs && ktiles <= 64;
  const DocTile* kd = a.k_tiles + (size_t)b * ktiles;
  DocTile dt = {0, -1, 0, 0};
  if (in_lanes && l < ktiles) dt = kd[l];
  const int pos = qi + p0;
  int qd = 0;
  // keys 0 .. jlim are allowed (but for documents); a row that does not exist
  // allows all, so that it asks for no mask
  int jlim = n - 1;
  if (valid) {
    if (a.causal) jlim = min(jlim, max(pos, a.prefix ? a.prefix[b] - 1 : -1));
    if (a.q_doc) {
      // (a row of no document needs no mask: it is written as one without keys)
      qd = a.q_doc[(size_t)b * a.Nq + qi];
      if (qd < 0) {
        valid = false;
        jlim = n - 1;
      }
    }
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
  const bool busy = jtop >= 0;  // this wavefront has a row with keys
  if (tid == 0) bad_pages = 0;
  // last key and smallest and largest document of the workgroup's rows
  int jend = jtop, lo = qlo, hi = qhi;
  if constexpr (!FEW) {
    if (l == 0) {
      red[w] = jtop;
      red[NW + w] = qlo;
      red[2 * NW + w] = qhi;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      jend = max(jend, red[i]);
      lo = min(lo, red[NW + i]);
      hi = max(hi, red[2 * NW + i]);
    }
  }
  int tbeg = 0, tend = (jend + 32) >> 5;
  if (docs && tend > 0) {
    // key tiles whose ids overlap those of the workgroup's rows: the first and the last
    int first, last;
    if (in_lanes) {
      const uint64_t m = __ballot(l < tend && dt.lo <= hi && dt.hi >= lo);
      first = m ? __builtin_ctzll(m) : tend;
      last = m ? 63 - __builtin_clzll(m) : -1;
    } else {
      doc_range<NW>(kd, tend, lo, hi, red, first, last);
    }
    tbeg = first;
    tend = last + 1;
  }
  if (it.part >= 0) dense_part(it.part, a.split.n, tbeg, tend);
  tbeg = uniform(tbeg);
  tend = uniform(tend);

  const float slope = MOD && a.slopes && valid ? a.slopes[hq] : 0.0f;
  const float sl2 = MOD ? 1.4426950408889634f : a.scale * 1.4426950408889634f;

  int pbase = 0;
  if constexpr (F8) {
    // pages of this workgroup's tiles
    pbase = (tbeg << 5) >> a.page_shift;
    const int pn = tend > tbeg ? ((((tend << 5) - 1) >> a.page_shift) - pbase + 1) : 0;
    __syncthreads();
    for (int i = tid; i < pn; i += 64 * NW) {
      const int at = pbase + i;
      int id = at < a.max_pages && (at << a.page_shift) < n ? a.table[(size_t)b * a.max_pages + at] : 0;
      if ((unsigned)id >= (unsigned)a.n_pages) {
        bad_pages = 1;
        if (a.status) atomicOr(a.status, ST_BAD_PAGE);
        id = -1;
      }
      const size_t e = (size_t)max(id, 0) * a.Hkv + hk;
      ptab[i] = make_int2(id, (uint16_t)((uint8_t)a.k_exp[e] | (uint8_t)a.v_exp[e] << 8));
    }
    __syncthreads();
  }
  const bool anybad = F8 && bad_pages;
  auto exp2i = [](int e) {
    return __uint_as_float((uint32_t)(min(max(e, CACHE_EMIN), CACHE_EMAX) + 127) << 23);
  };
  auto kscale = [&](int t) {  // power of two of this lane's key row
    if constexpr (F8) return exp2i((int8_t)ptab[((t * 32 + c32) >> a.page_shift) - pbase].y);
    else return 1.0f;
  };
  auto vscale = [&](int key) {
    if constexpr (F8) return exp2i((int8_t)(ptab[(key >> a.page_shift) - pbase].y >> 8));
    else return 1.0f;
  };

  if constexpr (FEW) dense_part(w, NW, tbeg, tend);  // this wavefront's own

  // Tiles [mlo, mhi) are allowed whole for every row of the wavefront.
  int mlo = tbeg, mhi = min((jfull + 1) >> 5, tend);
  if (docs) {
    int end = 0;
    if (in_lanes) {
      const uint64_t m = __ballot(qlo == qhi && l >= tbeg && l < tend && dt.uni && dt.lo == qlo);
      if (m) {
        mlo = __builtin_ctzll(m);
        const uint64_t run = m >> mlo;
        end = (run & (run + 1)) == 0 ? mlo + __builtin_popcountll(m) : 0;
      }
    } else {
      doc_run(kd, tbeg, tend, qlo == qhi ? qlo : -1, mlo, end);
    }
    mhi = min(mhi, end);
  }
  if (anybad) mhi = 0;

  // Copies of the tiles in order, K and V each with a place in memory, a ring
  // slot and a lane offset that only the last, partial tile changes.
  struct Feed {
    const char* src;  // first row of the next tile
    uint32_t slot, lane;
  };
  auto lane_off = [&](int64_t rs) { return (uint32_t)((l >> 2) * rs) + TL::copy_byte(0, l); };
  Feed fk = {F8 ? a.k.p : a.k.p + b * a.k.b + hk * a.k.h + (int64_t)tbeg * 32 * a.k.r, 0,
             F8 ? (l >> 2) * D + TL::copy_byte(0, l) : lane_off(a.k.r)};
  Feed fv = {F8 ? a.v.p : a.v.p + b * a.v.b + hk * a.v.h + (int64_t)tbeg * 32 * a.v.r, 0,
             F8 ? fk.lane : lane_off(a.v.r)};
  auto next = [](uint32_t& slot) {
    const uint32_t now = slot;
    slot = (slot + TL::BYTES) & (RING - 1);
    return now;
  };
  static_assert((RING & (RING - 1)) == 0, "ring size");
  // whole: all rows of the tile exist
  auto issue = [&](auto whole, Feed& f, int64_t rs, int t, uint32_t ring) {
    const uint32_t to = ring + next(f.slot);
    bool copies = true;
    if constexpr (!FEW && TL::DW < 4) copies = w < TL::DW;
    if (copies) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int c = FEW ? i : w * NI + i;
        if constexpr (F8) {
          // (the 16 rows of one copy lie in one page)
          const int row = t * 32 + 16 * (c & 1);
          const int id = uniform(ptab[(row >> a.page_shift) - pbase].x);
          const int in = row & ((1 << a.page_shift) - 1);
          const size_t at = ((((size_t)max(id, 0) * a.Hkv + hk) << a.page_shift) + in) * D;
          lds_dma16(f.src + at + 64 * (c >> 1), f.lane, to + 1024 * c);
        } else if (whole.value || 32 * t + 32 <= n) {
          lds_dma16(f.src + 16 * (c & 1) * rs + 64 * (c >> 1), f.lane, to + 1024 * c);
        } else {  // rows past the last: the last
          const int64_t row = min(TL::copy_row(c, l), n - 1 - 32 * t);
          lds_dma16(f.src, (uint32_t)(row * rs) + TL::copy_byte(c, l), to + 1024 * c);
        }
      }
    }
    if constexpr (!F8) f.src += 32 * rs;
  };
  // documents of the keys of tiles t and t + 1 (a pair; past the last: the last)
  auto issue_docs = [&](int t) {
    if (docs && w == 0 && t < tend)
      lds_dma4(a.k_doc + (size_t)b * a.Nk, 4 * (uint32_t)min(32 * t + l, n - 1),
               lds_addr(kds[((t - tbeg) >> 1) & 3]));
  };
  auto issue_k = [&](int t) { issue(std::false_type{}, fk, a.k.r, t, kt); };
  auto issue_v = [&](int t) { issue(std::false_type{}, fv, a.v.r, t, vt); };

  float m = DENSE_NOKEY, lsum = 0.0f, tmax = DENSE_NOKEY;
  f32x16_t acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x16_t{};

  // operands of a tile's scores
  using raw = typename DenseOp<T>::raw;
  raw kf[F32 ? 1 : KS];
  float ke = 1.0f;
  uint32_t ks = 0, kread = 0, vread = 0;
  const uint32_t krow = kt + TL::row_at(l), vcol = vt + TL::col_at(l);
  auto load_k = [&](int t) {  // (the tiles in order)
    ks = next(kread) + krow;
    if constexpr (F8) ke = kscale(min(t, tend - 1));
    if constexpr (!F32) {
#pragma unroll
      for (int s = 0; s < KS; ++s) kf[s] = dense_row_raw<T, D>(ks, s);
    }
  };
  // (float: its products are slow enough to read each operand when it is used)
  auto k_frag = [&](int s) {
    if constexpr (F32) return dense_row_raw<T, D>(ks, s);
    else return dense_cvt<T>(kf[s], ke);
  };
  auto page_of = [&](int j) {
    return F8 ? ptab[(min(j, 32 * tend - 1) >> a.page_shift) - pbase].x : 0;
  };
  // variants, masks and row maxima of tile t's scores
  uint32_t okn = 0u;  // allowed pairs of the tile whose scores were finished last (if masked)
  auto finish = [&](auto masked, int t, f32x16_t& st) {
    if constexpr (MOD) {
      if (a.cap > 0.0f) {
        dense_cap_tile<false>(st, a, nullptr);
      } else {
#pragma unroll
        for (int q = 0; q < 16; ++q) st[q] *= a.scale;
      }
      if (a.slopes) {
        const float far = (float)(pos - 32 * t - 4 * hf);
#pragma unroll
        for (int q = 0; q < 16; ++q)
          st[q] = fmaf(-slope, fabsf(far - (float)(8 * (q >> 2) + (q & 3))), st[q]);
      }
    }
    if (masked.value && (t < mlo || t >= mhi)) {
      // (rare, and kept from being prepared outside the loop)
      const int j0 = opaque(32 * t + 4 * hf);
      uint32_t bits = 0u;
#pragma unroll
      for (int q = 0; q < 16; ++q) bits |= bit_ge0(jlim - j0 - 8 * (q >> 2) - (q & 3)) << q;
      if (docs && FEW) {
        const int* kd = a.k_doc + (size_t)b * a.Nk;
#pragma unroll
        for (int q = 0; q < 16; ++q)
          bits &= ~(bit_ne0(kd[min(j0 + 8 * (q >> 2) + (q & 3), n - 1)] ^ qd) << q);
      } else if (docs) {
        const int i = t - tbeg, *kd = &kds[(i >> 1) & 3][32 * (i & 1) + 4 * hf];
#pragma unroll
        for (int q = 0; q < 16; ++q) bits &= ~(bit_ne0(kd[8 * (q >> 2) + (q & 3)] ^ qd) << q);
      }
      if (anybad) {
#pragma unroll
        for (int q = 0; q < 16; ++q)
          bits &= ~((1u - bit_ge0(page_of(j0 + 8 * (q >> 2) + (q & 3)))) << q);
      }
#pragma unroll
      for (int q = 0; q < 16; ++q) st[q] = mask_score(st[q], bits, q);
      okn = bits;
    }
    float x = st[0];
#pragma unroll
    for (int q = 1; q < 16; ++q) x = fmaxf(x, st[q]);
    tmax = max_xor32(x);
  };
  // One step of the pipeline.  At the top: sc holds the scores of tile t and
  // tmax their row maxima, kf the operands of tile t + 1's.  LDS reads are issued
  // half a step before their use and the vector work sits between the MFMAs:
  //   first half   S(t+1) = K Q^T        beside the probabilities of tile t
  //   second half  O += V(t)^T P(t)^T    beside the row maxima of tile t + 1
  // (scores past the last tile come from a stale slot and are never used)
  // masked: tile t or tile t + 1 may have pairs that are not allowed
  //
  // Tiles arrive in pairs, one barrier for 64 keys: before the first step of a
  // pair, K up to t + KA + 1 and V up to t + 1 have landed, and the next pair is
  // asked for, into the slots that the pair before has been read from.  With
  // rings of their own (FEW) wavefronts wait and ask tile by tile, up to
  // K(t + 3), V(t + 2) in flight: there the copies in flight are what counts.
  // sure: the tiles to be asked for exist and are whole
  auto arrive = [&](auto sure, int t) {
    if constexpr (FEW) {
      // K(t+KA) and all before it (V(t)) has landed; V(t+1), K(t+KA+1), V(t+2) may stay
      if (t + KA + 1 < tend) wait_vmcnt<3 * NI>();
      else wait_vmcnt<0>();
    } else if (((t - tbeg) & 1) == 0) {
      wait_vmcnt<0>();
      __syncthreads();
      if constexpr (!F8) issue_docs(t + 4);
      if constexpr (sure.value) {
        issue(sure, fk, a.k.r, t + KA + 2, kt);
        issue(sure, fv, a.v.r, t + 2, vt);
        issue(sure, fk, a.k.r, t + KA + 3, kt);
        issue(sure, fv, a.v.r, t + 3, vt);
      } else {
        if (t + KA + 2 < tend) issue_k(t + KA + 2);
        if (t + 2 < tend) issue_v(t + 2);
        if (t + KA + 3 < tend) issue_k(t + KA + 3);
        if (t + 3 < tend) issue_v(t + 3);
      }
    }
  };
  auto ask = [&](int t) {
    if constexpr (FEW) {
      if (t + KA + 2 < tend) issue_k(t + KA + 2);
      if (t + 3 < tend) issue_v(t + 3);
    }
  };
  auto step = [&](auto masked, auto sure, int t, const f32x16_t& sc, f32x16_t& sn) {
    arrive(sure, t);
    const uint32_t okc = okn;
    // a row's reference moves only when its maximum exceeds it by more than 2^8 in
    // probability, whatever the wavefront's other rows do (their contents are not
    // to change its rounding)
    const bool up = (tmax - m) * sl2 > 8.0f;
    if (__any(up)) {
      const float mnew = up ? tmax : m;
      const float alpha = __builtin_amdgcn_exp2f((m - mnew) * sl2);
      lsum *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] *= alpha;
      m = mnew;
    }
    const uint32_t vs = next(vread) + vcol;
    raw vf[2][DB];
    float ve[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      ve[kk] = vscale(32 * t + 16 * kk);
#pragma unroll
      for (int db = 0; db < DB; ++db) vf[kk][db] = dense_col_raw<T, D>(vs, kk, db);
    }
    frag vc[2][DB];
    if constexpr (masked.value) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int db = 0; db < DB; ++db) vc[kk][db] = dense_cvt<T>(vf[kk][db], ve[kk]);
      if (t < mlo || t >= mhi) {
        // a value that is not finite is read by the rows that allow its key only
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          frag f[2] = {vc[0][db], vc[1][db]};
          dense_guard(f, okc, acc[db]);
          vc[0][db] = f[0];
          vc[1][db] = f[1];
        }
      }
    }
    f32x16_t p;
    float ls[2] = {0.0f, 0.0f};
    const float nms = -m * sl2;
    constexpr int EP = 16 / KS;  // scores per product of the first half
    sn = f32x16_t{};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      sn = dense_mma(k_frag(s), qf[s], sn);
#pragma unroll
      for (int e = EP * s; e < EP * (s + 1); ++e) {
        // (float: the difference first, so that the rounding is relative to it)
        p[e] = __builtin_amdgcn_exp2f(F32 ? (sc[e] - m) * sl2 : fmaf(sc[e], sl2, nms));
        ls[e & 1] += p[e];
      }
      // (the sums are taken here, so that the probabilities need not be kept)
      asm volatile("" : "+v"(ls[0]), "+v"(ls[1]));
    }
    lsum += ls[0] + ls[1];
    frag pf[2];
    dense_pack(pf[0], p, 0);
    dense_pack(pf[1], p, 1);
    load_k(t + 2);
    if constexpr (!masked.value) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int db = 0; db < DB; ++db) vc[kk][db] = dense_cvt<T>(vf[kk][db], ve[kk]);
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] = dense_mma(vc[kk][db], pf[kk], acc[db]);
    finish(masked, t + 1, sn);
    ask(t);
  };
  if (tbeg < tend) {
    // fill: K(0) .. K(KA+1), V(0), V(1); S(0), the operands of S(1)
    f32x16_t s0 = {}, s1;
    // (the queries have arrived: from here on the counted waits see only the copies)
#pragma unroll
    for (int s = 0; s < KS; ++s) dense_arrived(qf[s]);
    if constexpr (!FEW && !F8) {
      issue_docs(tbeg);
      issue_docs(tbeg + 2);
    }
    issue_k(tbeg);
    if (tbeg + 1 < tend) issue_k(tbeg + 1);
    issue_v(tbeg);
    if (KA > 1 && tbeg + 2 < tend) issue_k(tbeg + 2);
    if (tbeg + 1 < tend) issue_v(tbeg + 1);
    // K(0), K(1) (V(0), K(2), V(1) may stay)
    if (tbeg + 2 < tend) wait_vmcnt<(KA > 1 ? 3 : 2) * NI>();
    else wait_vmcnt<0>();
    if constexpr (!FEW) __syncthreads();
    if (busy) {
      load_k(tbeg);
#pragma unroll
      for (int s = 0; s < KS; ++s) s0 = dense_mma(k_frag(s), qf[s], s0);
      load_k(tbeg + 1);
      finish(std::true_type{}, tbeg, s0);
    }
    if (tbeg + KA + 1 < tend) issue_k(tbeg + KA + 1);
    if (FEW && tbeg + 2 < tend) issue_v(tbeg + 2);
    int t = tbeg;
    if (!busy) {  // (its share of the copies only)
      for (; t < tend; ++t) {
        arrive(std::false_type{}, t);
        ask(t);
      }
    }
    while (t < tend) {
      // most tiles: no masking in the loop
      auto plain = [&](int t) { return t >= mlo && t + 2 < mhi && (FEW || ((t - tbeg) & 1) == 0); };
      if constexpr (!FEW) {
        for (; plain(t) && t + KA + 3 < mhi; t += 2) {
          step(std::false_type{}, std::true_type{}, t, s0, s1);
          step(std::false_type{}, std::true_type{}, t + 1, s1, s0);
        }
      }
      for (; plain(t); t += 2) {
        step(std::false_type{}, std::false_type{}, t, s0, s1);
        step(std::false_type{}, std::false_type{}, t + 1, s1, s0);
      }
      if (t >= tend) break;
      step(std::true_type{}, std::false_type{}, t, s0, s1);
      s0 = s1;
      ++t;
    }
  }

  lsum += __shfl_xor(lsum, 32, 64);
  if (!valid) {  // (a row of no document)
    m = DENSE_NOKEY;
    lsum = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = f32x16_t{};
  }
  const bool staged = !FEW && !a.out_f32 && it.part < 0;
  if (staged) __syncthreads();  // (the rings are done with)
  if constexpr (FEW && NW > 1) {
    // the parts of a row joined in LDS, wavefront by wavefront in order
    constexpr int PS = D + 4;  // (4 floats of padding against bank conflicts)
    static_assert((size_t)NW * 32 * PS * 4 <= NW * dense_ring<T, D>(), "room for the parts");
    __shared__ float2 ml[NW][32];
    float* part = (float*)smem;
    if (hf == 0) ml[w][c32] = make_float2(m, lsum);
    __syncthreads();  // (and every ring is done with)
    float mall = ml[0][c32].x, lall = 0.0f;
#pragma unroll
    for (int i = 1; i < NW; ++i) mall = fmaxf(mall, ml[i][c32].x);
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float2 y = ml[i][c32];
      lall += y.y == 0.0f ? 0.0f : y.y * __builtin_amdgcn_exp2f((y.x - mall) * sl2);
    }
    const float fac = lsum == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((m - mall) * sl2);
    if (exists) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q = 0; q < 16; q += 4)
          *(float4*)(part + (w * 32 + c32) * PS + 32 * db + 2 * q + 4 * hf) =
              make_float4(acc[db][q] * fac, acc[db][q + 1] * fac, acc[db][q + 2] * fac,
                          acc[db][q + 3] * fac);
    }
    __syncthreads();
    // (this wavefront adds and writes its share of the columns)
    m = mall;
    lsum = lall;
#pragma unroll
    for (int db = 0; db < DB; ++db)
      if (db % NW == w) {
#pragma unroll
        for (int q = 0; q < 16; q += 4) {
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int i = 0; i < NW; ++i) {
            const float4 y = *(const float4*)(part + (i * 32 + c32) * PS + 32 * db + 2 * q + 4 * hf);
            x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
          }
          acc[db][q] = x.x, acc[db][q + 1] = x.y, acc[db][q + 2] = x.z, acc[db][q + 3] = x.w;
        }
      }
  }
  auto mine = [&](int db) { return !FEW || db % NW == w; };
  if (it.part >= 0) {
    if (!exists) return;
    const size_t row = (size_t)it.slot * ROWS + (FEW ? 0 : 32 * w) + c32;
    if (hf == 0 && mine(0)) a.ml[row] = make_float2(m, lsum);
    float* o = a.part + row * D + 4 * hf;
#pragma unroll
    for (int db = 0; db < DB; ++db)
      if (mine(db)) {
#pragma unroll
        for (int q = 0; q < 16; q += 4)
          *(float4*)(o + 32 * db + 2 * q) =
              make_float4(acc[db][q], acc[db][q + 1], acc[db][q + 2], acc[db][q + 3]);
      }
    return;
  }
  // (a row without a key: zeros; a sum that is not a number stays one)
  const float inv = lsum == 0.0f ? 0.0f : 1.0f / lsum;
  if (a.lse && hf == 0 && exists && mine(0))
    a.lse[((size_t)b * a.Hkv * a.G + hq) * a.Nq + qi] =
        lsum == 0.0f ? -INFINITY : m * (MOD ? 1.0f : a.scale) + logf(lsum);
  if (staged) {
    // through LDS, so that a row's 16 bytes a lane leave side by side
    constexpr int LPR = D / 8, RS = 2 * D + 16;  // lanes and padded bytes of a row
    unsigned char* st = smem + w * 32 * RS;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q = 0; q < 16; q += 4)
        *(uint2*)(st + c32 * RS + 2 * (32 * db + 2 * q + 4 * hf)) =
            make_uint2(pack_bf(acc[db][q] * inv, acc[db][q + 1] * inv),
                       pack_bf(acc[db][q + 2] * inv, acc[db][q + 3] * inv));
#pragma unroll
    for (int i = 0; i < 32 / (64 / LPR); ++i) {
      const int row = i * (64 / LPR) + l / LPR, c = l % LPR;
      const int ri = __shfl(exists ? qi : -1, row, 64), rh = __shfl(hq, row, 64);
      const uint4 x = *(const uint4*)(st + row * RS + 16 * c);
      if (ri >= 0) *(uint4*)(a.o.p + b * a.o.b + rh * a.o.h + ri * a.o.r + 16 * c) = x;
    }
    return;
  }
  if (!exists) return;
  char* o = a.o.p + b * a.o.b + hq * a.o.h + qi * a.o.r;
#pragma unroll
  for (int db = 0; db < DB; ++db)
    if (mine(db)) {
#pragma unroll
      for (int q = 0; q < 16; q += 4) {
        const int c = 32 * db + 2 * q + 4 * hf;
        const float x0 = acc[db][q] * inv, x1 = acc[db][q + 1] * inv, x2 = acc[db][q + 2] * inv,
                    x3 = acc[db][q + 3] * inv;
        if (a.out_f32) store_out4<float>((float*)o + c, x0, x1, x2, x3);
        else store_out4<bf16_t>((bf16_t*)o + c, x0, x1, x2, x3);
      }
    }
}

// The parts of a row joined: O = sum_s 2^(m_s - m) acc_s / sum_s 2^(m_s - m) l_s
// in the parts' order, by D / 4 lanes of four columns each, with four parts' loads
// in flight.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void k_dense_join(const DenseArgs a, float sl2) {
  constexpr int L = D / 4;
  const int row = blockIdx.x * (256 / L) + threadIdx.x / L, l = threadIdx.x % L;
  const int rows = a.split.rest * ROWS, nrt = (a.R + ROWS - 1) / ROWS, heads = a.B * a.Hkv;
  if (row >= rows) return;
  const int unit = a.split.whole + row / ROWS;  // (as dense_item has them)
  const int bh = a.causal ? unit % heads : unit / nrt;
  const int rt = nrt - 1 - (a.causal ? unit / heads : unit % nrt);
  const int r = rt * ROWS + row % ROWS, b = bh / a.Hkv;
  const int qi = r / a.G, hq = bh % a.Hkv * a.G + r % a.G;
  if (r >= a.R || (a.q_lens && qi >= min(max(a.q_lens[b], 0), a.Nq))) return;
  const float2* ml = a.ml + row;
  const float* part = a.part + (size_t)row * D + 4 * l;
  float m = DENSE_NOKEY;
  for (int i = l; i < a.split.n; i += L) m = fmaxf(m, ml[(size_t)i * rows].x);
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, L));
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.0f;
#pragma unroll 4
  for (int i = 0; i < a.split.n; ++i) {
    const float2 s = ml[(size_t)i * rows];
    const float4 p = *(const float4*)(part + (size_t)i * rows * D);
    if (s.y == 0.0f) continue;  // (no key of its own)
    const float f = __builtin_amdgcn_exp2f((s.x - m) * sl2);
    sum = fmaf(f, s.y, sum);
    x.x = fmaf(f, p.x, x.x), x.y = fmaf(f, p.y, x.y);
    x.z = fmaf(f, p.z, x.z), x.w = fmaf(f, p.w, x.w);
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  if (a.lse && l == 0)
    a.lse[((size_t)b * a.Hkv * a.G + hq) * a.Nq + qi] =
        sum == 0.0f ? -INFINITY : m * (sl2 * 0.69314718055994531f) + logf(sum);
  char* o = a.o.p + b * a.o.b + hq * a.o.h + qi * a.o.r;
  if (a.out_f32)
    store_out4<float>((float*)o + 4 * l, x.x * inv, x.y * inv, x.z * inv, x.w * inv);
  else
    store_out4<bf16_t>((bf16_t*)o + 4 * l, x.x * inv, x.y * inv, x.z * inv, x.w * inv);
}

// A chip of 256 CUs runs 256 per_cu workgroups at a time, a round.  Whole rounds
// take tiles whole; what is left, or all of a launch that fills no round, is cut
// into parts of at least 8 streamed tiles (2 for float).  Where the lengths
// differ, three rounds of parts.  Else as many as give the least time, counted in
// streamed tiles (about 1 us a round; float 16): the rounds of parts, a round's
// sums written and read again (14; 1), and the launch that joins them; it has to
// save a tenth.  (Against as many parts as fit one round: 9 float heads of 4096
// rows 366 us instead of 536, their gradient 1451 instead of 2294; 32 heads of
// 512, where two parts a tile do not pay, 15.2 instead of 24.6.  6 heads of 8192
// as three rounds of quarters take 237 us, whole 226.)  With a causal mask the last tiles are the
// short ones, and only a launch of less than a round is cut.
DenseSplit dense_split(int64_t held, int64_t tiles, bool f32, bool uneven, bool causal, int per_cu,
                       int launch) {
  const int64_t slots = 256 * per_cu, least = f32 ? 2 : 8;
  const int64_t rest = held < slots ? held : causal ? 0 : held % slots;
  int64_t n = 1;
  const int64_t most = std::min<int64_t>(tiles / least, DENSE_MAXSPLIT);
  if (rest > 0 && (uneven || causal)) {
    n = std::min(3 * slots / rest, most);
  } else if (rest > 0) {
    double best = 0.9 * tiles;
    for (int64_t k = 2; k <= most; ++k) {
      const int64_t rounds = (rest * k + slots - 1) / slots;
      const double sums = (f32 ? 1.0 : 14.0) * (rest * k) / slots + (f32 ? 1.0 : launch);
      const double time = rounds * ((tiles + k - 1) / k) + sums;
      if (time < best) best = time, n = k;
    }
  }
  if (n > 1) return {(int)(held - rest), (int)rest, (int)n};
  return {(int)held, 0, 1};
}

// key tiles a part of the form for few rows has at least: eight a wavefront (at
// one query over 1000 keys parts of two took as long as the launch that joins
// them costs)
template <class T, int D>
constexpr int few_least() { return 8 * dense_few_waves<T, D>(); }

DenseSplit dense_fwd_split(int64_t rows, int64_t heads, int64_t key_tiles, int d, int dtype, bool cached,
                           bool uneven, bool causal) {
  if (rows > DENSE_FEW)
    return dense_split((rows + DENSE_ROWS - 1) / DENSE_ROWS * heads, key_tiles,
                       !cached && dtype == PARK_F32, uneven, causal, cached && d == 64 ? 3 : 2, 6);
  const int least = cached ? (d == 128 ? few_least<fp8_t, 128>() : few_least<fp8_t, 64>())
                    : dtype == PARK_BF16 ? (d == 128 ? few_least<bf16_t, 128>() : few_least<bf16_t, 64>())
                                         : (d == 128 ? few_least<float, 128>() : few_least<float, 64>());
  const int64_t held = rows > 0 ? heads : 0;
  const int64_t n = std::min<int64_t>(std::min<int64_t>(held ? 1024 / held : 1, key_tiles / least),
                                      DENSE_MAXSPLIT);
  if (n > 1) return {0, (int)held, (int)n};
  return {(int)held, 0, 1};
}

template <class T, int D, bool MOD, bool FEW>
static park_status fwd_launch(const DenseArgs& a, hipStream_t st) {
  constexpr int NW = FEW ? dense_few_waves<T, D>() : 4, rows = FEW ? 32 : DENSE_ROWS;
  constexpr size_t lds =
      (FEW ? NW : 1) * dense_ring<T, D>() + (sizeof(T) == 1 ? DENSE_PAGES * sizeof(int2) : 0);
  static std::atomic<uint64_t> done{0};
  PARK_TRY(reserve_lds((const void*)k_dense_fwd<T, D, MOD, FEW>, lds, done, "dense attention"));
  PARK_LAUNCH(FEW ? "dense_fwd_few" : "dense_fwd", (k_dense_fwd<T, D, MOD, FEW>),
              dim3((unsigned)a.split.groups()), dim3(64 * NW), lds, st, a);
  if (a.split.rest) {
    const float sl2 = (MOD ? 1.0f : a.scale) * 1.4426950408889634f;
    PARK_LAUNCH("dense_join", (k_dense_join<D, rows>), dim3(a.split.rest * (rows * (D / 4) / 256)),
                dim3(256), 0, st, a, sl2);
  }
  return PARK_OK;
}

template <class T, int D, bool MOD>
static park_status fwd_form(const DenseArgs& a, hipStream_t st) {
  return a.R <= DENSE_FEW ? fwd_launch<T, D, MOD, true>(a, st) : fwd_launch<T, D, MOD, false>(a, st);
}

template <class T>
static park_status fwd_type(const DenseArgs& a, int d, hipStream_t st) {
  const bool mod = a.cap > 0.0f || a.slopes;
  if (d == 128) return mod ? fwd_form<T, 128, true>(a, st) : fwd_form<T, 128, false>(a, st);
  return mod ? fwd_form<T, 64, true>(a, st) : fwd_form<T, 64, false>(a, st);
}

park_status launch_dense_fwd(const DenseArgs& a, int d, int dtype, bool cached, hipStream_t st) {
  if (cached) return fwd_type<fp8_t>(a, d, st);
  return dtype == PARK_BF16 ? fwd_type<bf16_t>(a, d, st) : fwd_type<float>(a, d, st);
}

}  // namespace park
