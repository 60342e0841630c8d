// Writing the 8-bit key/value cache.
//
// A page holds `page` consecutive tokens of a sequence for each key/value head
// as e4m3 values q and one exponent e for the page and head: the value is
// q 2^e.  e is the smallest exponent with max |x| <= 448 2^e over the tokens
// written so far (a power of two costs e4m3, a floating format, no precision
// above its subnormals).  New tokens in a page that has older ones may raise
// e; the older values are then rounded again, which changes only those that
// become subnormal.
//
// Memory bound: one workgroup per touched page, head and side reads the new
// rows once, keeps them in registers across the maximum, and writes them; the
// older rows are read only if e rises.  4 sequences of 8192 new tokens, 8 heads of
// 128: 30 us = 4.2 TB/s (a large copy: 4.86); one token each of 64 sequences:
// 4.9 us (a call from Python takes 13).
#include "dense.h"
#include "kernels.h"

namespace park {

__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// eight floats as e4m3 (round to nearest even; NaN for what is not finite or rounds
// past 448)
__device__ __forceinline__ uint2 to_f8(const float* x, float s) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int p = 0;
    p = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * s, x[4 * i + 1] * s, p, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * s, x[4 * i + 3] * s, p, true);
    w[i] = (uint32_t)p;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((__float_as_uint(x[4 * i + k]) & 0x7f800000u) == 0x7f800000u)
        w[i] = (w[i] & ~(0xffu << (8 * k))) | 0x7fu << (8 * k);
  }
  return make_uint2(w[0], w[1]);
}

// C: pieces of 8 elements a thread holds (page * d <= 2048 C)
template <class T, int C>
__global__ __launch_bounds__(256) void k_cache_append(const CacheAppend a, int slots) {
  __shared__ float red[4];
  const int tid = threadIdx.x;
  int item = blockIdx.x;
  const int hk = item % a.Hkv;
  item /= a.Hkv;
  const int slot_i = item % slots, b = item / slots;
  const int page = 1 << a.page_shift;
  const int len = max(a.lens[b], 0), add = a.n_new ? min(max(a.n_new[b], 0), a.N) : a.N;
  const int slot = (len >> a.page_shift) + slot_i;
  const int64_t first = (int64_t)slot << a.page_shift, end = (int64_t)len + add;
  if (add == 0 || first >= end) return;
  const int id = slot < a.max_pages ? a.table[(size_t)b * a.max_pages + slot] : -1;
  if ((unsigned)id >= (unsigned)a.n_pages) {
    if (a.status && tid == 0) atomicOr(a.status, ST_BAD_PAGE);
    return;
  }
  const RowsArg x = blockIdx.y ? a.v : a.k;
  const size_t block = (size_t)id * a.Hkv + hk;
  uint8_t* pool = (blockIdx.y ? a.pv : a.pk) + block * page * a.d;
  int8_t* exps = (blockIdx.y ? a.v_exp : a.k_exp) + block;
  const int r0 = (int)max(len - first, (int64_t)0), r1 = (int)min(end - first, (int64_t)page);
  const char* src = x.p + b * x.b + hk * x.h + (first - len) * x.r;
  const int dshift = a.d == 128 ? 7 : 6;

  // this thread's pieces: the new rows' elements, and their largest magnitude
  float v[C][8];
  float top = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int e = (c * 256 + tid) * 8, row = e >> dshift, col = e & (a.d - 1);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[c][k] = 0.0f;
    if (row >= r0 && row < r1) {
      const char* p = src + row * x.r + col * sizeof(T);
      if constexpr (sizeof(T) == 4) {
        *(float4*)v[c] = *(const float4*)p;
        *(float4*)(v[c] + 4) = *(const float4*)(p + 16);
      } else {
        const uint4 u = *(const uint4*)p;
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[c][2 * k] = bf2f((bf16_t)w[k]);
          v[c][2 * k + 1] = bf2f((bf16_t)(w[k] >> 16));
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float y = fabsf(v[c][k]);
        top = fmaxf(top, y < INFINITY ? y : 0.0f);
      }
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  if ((tid & 63) == 0) red[tid >> 6] = top;
  const int e_old = min(max((int)*exps, CACHE_EMIN), CACHE_EMAX);
  __syncthreads();  // (every thread has read the exponent)
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  // top = 1.f 2^E; 448 = 1.75 2^8
  const uint32_t u = __float_as_uint(top);
  int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  e = min(max(e, CACHE_EMIN), CACHE_EMAX);
  if (r0 > 0) e = max(e, e_old);
  const bool again = r0 > 0 && e > e_old;
  const float s = pow2i(-e), down = pow2i(max(e_old - e, -126));
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * 256 + tid) * 8, row = at >> dshift;
    if (row >= r0 && row < r1) {
      *(uint2*)(pool + at) = to_f8(v[c], s);
    } else if (again && row < r0) {
      const uint2 w = *(const uint2*)(pool + at);
      const uint4 y = __builtin_bit_cast(uint4, cvt_f8x8(u32x2_t{w.x, w.y}, 1.0f));
      const uint32_t z[4] = {y.x, y.y, y.z, y.w};
      float f[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        f[2 * k] = bf2f((bf16_t)z[k]);
        f[2 * k + 1] = bf2f((bf16_t)(z[k] >> 16));
      }
      *(uint2*)(pool + at) = to_f8(f, down);
    }
  }
  if (tid == 0) *exps = (int8_t)e;
}

template <class T, int C>
static park_status append_launch(const CacheAppend& a, hipStream_t st) {
  const int page = 1 << a.page_shift;
  const int slots = (int)(((int64_t)a.N + 2 * page - 2) / page);
  PARK_LAUNCH("cache_append", (k_cache_append<T, C>),
              dim3((unsigned)((int64_t)a.B * slots * a.Hkv), 2), dim3(256), 0, st, a, slots);
  return PARK_OK;
}

template <class T>
static park_status append_type(const CacheAppend& a, hipStream_t st) {
  const int n = a.d << a.page_shift;
  if (n <= 2048) return append_launch<T, 1>(a, st);
  if (n <= 4096) return append_launch<T, 2>(a, st);
  if (n <= 8192) return append_launch<T, 4>(a, st);
  return append_launch<T, 8>(a, st);
}

park_status launch_cache_append(const CacheAppend& a, hipStream_t st) {
  return a.dtype == PARK_BF16 ? append_type<bf16_t>(a, st) : append_type<float>(a, st);
}

}  // namespace park
