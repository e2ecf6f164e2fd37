// cache_write, cache_read: rows of K and V into the quantised cache and out of it.
//
// A thread holds 8 channels of a row of K and the same of V (d / 8 threads a row), four threads share a scale.  The scale is the least
// power of two at which the group's largest value lies no further than half a step beyond the largest code (7 for e2m1, 464 for
// e4m3), so the largest value is rounded as any other is (e2m1 on Gaussian groups: off by 0.112 of the 2-norm; with that border at 6 or
// at 8 it is 0.115).  All of it is exact in fp32: the exponent comes from the bits of the largest value, and a product with a power
// of two does not round; codes are rounded to nearest, ties to even.
//
// What bounds them: memory.  Rows go in token order within a head, so the codes of neighbouring threads lie side by side.  12 heads of 4680 rows
// of 128 channels in 8 bits, 43.6 MB each way: written in 11 us, read in 9; 2 x 12 heads of 14047 rows from 4 bits, 218 MB: 35 us.  One row
// for each of 32 sequences: 3.6 and 3.1 us, a launch and two dependent round trips.
#include "usv_attn_bf16.h"
#include "usv_cache.h"

namespace usv {
namespace {

typedef __attribute__((__vector_size__(2 * sizeof(short)))) short s16x2;

template <int BITS>
struct Code;
template <>
struct Code<4> {
  static constexpr unsigned kRound = 0x1fffff, kTop = 2, kLeast = 2, kLast = 252;  // mantissas beyond 1.75 go up; exponent of the largest code
  static constexpr float kMost = 6.f;
};
template <>
struct Code<8> {
  static constexpr unsigned kRound = 0x17ffff, kTop = 8, kLeast = 10, kLast = 246;  // beyond 1.8125
  static constexpr float kMost = 448.f;
};

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const float4 a = bf16_pair(u.x, u.y), b = bf16_pair(u.z, u.w);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

// Where a row lies: false if it is not to be touched.
struct Place {
  int b, h, i;
  long long page;  // < 0: no such page
  int row;
};
__device__ __forceinline__ void place_at(const CacheRowsArgs& a, long long pos, Place* p) {
  p->page = -1, p->row = 0;
  if (pos >= 0 && pos < (long long)a.c.table_pages * a.c.page_size) {
    const int slot = (int)pos / a.c.by_page;
    p->row = (int)(pos - (long long)slot * a.c.page_size);
    const int page = a.c.table[(long long)p->b * a.c.table_pages + slot];
    if (page >= 0 && page < a.c.pages) p->page = page;
  }
}

template <int D>
__device__ __forceinline__ bool place_of(const CacheRowsArgs& a, Place* p) {
  constexpr int PER = D / 8;
  const long long i = (long long)blockIdx.x * (256 / PER) + threadIdx.x / PER;
  if (i >= a.rows) return false;
  p->i = (int)i, p->h = blockIdx.y, p->b = blockIdx.z;
  if (a.counts && p->i >= a.counts[p->b]) return false;
  place_at(a, (long long)a.starts[p->b] + p->i, p);
  return true;
}

template <typename T, int D, int BITS>
__global__ __launch_bounds__(256) void cache_write(CacheRowsArgs a) {
  constexpr int PER = D / 8, CB = D * BITS / 8, SB = D / 32;
  Place p;
  if (!place_of<D>(a, &p) || p.page < 0) return;
  const int t = threadIdx.x % PER;
  float x[2][8];
  load8(reinterpret_cast<const T*>(static_cast<const unsigned char*>(a.k) + p.b * a.sk.batch + p.h * a.sk.head + p.i * a.sk.token) + 8 * t, x[0]);
  load8(reinterpret_cast<const T*>(static_cast<const unsigned char*>(a.v) + p.b * a.sv.batch + p.h * a.sv.head + p.i * a.sv.token) + 8 * t, x[1]);
  unsigned char* base = a.cache + (p.page * a.c.H + p.h) * a.c.head_bytes();
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    unsigned top = 0;  // (as bits: an infinity or a NaN is larger than any number)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[which][e]) & 0x7fffffffu);
    top = max(top, (unsigned)__shfl_xor((int)top, 1));  // (the four threads of a group are in one row: all here or none)
    top = max(top, (unsigned)__shfl_xor((int)top, 2));
    int scale = (int)((top + Code<BITS>::kRound) >> 23) - (int)Code<BITS>::kTop;
    scale = top >= 0x7f800000u ? 255 : min(max(scale, (int)Code<BITS>::kLeast), (int)Code<BITS>::kLast);  // (no code stands for more than fp32 holds)
    const float inv = __uint_as_float((unsigned)max(254 - scale, 0) << 23);  // 2^-e
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = scale == 255 ? 0.f : fminf(fmaxf(x[which][e] * inv, -Code<BITS>::kMost), Code<BITS>::kMost);
    unsigned char* codes = base + (which * a.c.page_size + p.row) * (long long)CB + t * BITS;
    if constexpr (BITS == 4) {
      unsigned w = 0;
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.0f, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.0f, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.0f, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.0f, 3);
      *reinterpret_cast<unsigned*>(codes) = w;
    } else {
      s16x2 w0 = {0, 0}, w1 = {0, 0};
      w0 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w0, y[0], y[1], 1.0f, false);
      w0 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w0, y[2], y[3], 1.0f, true);
      w1 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w1, y[4], y[5], 1.0f, false);
      w1 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w1, y[6], y[7], 1.0f, true);
      *reinterpret_cast<uint2*>(codes) = make_uint2(__builtin_bit_cast(unsigned, w0), __builtin_bit_cast(unsigned, w1));
    }
    if ((t & 3) == 0)
      base[2LL * a.c.page_size * CB + ((long long)which * a.c.page_size + p.row) * SB + t / 4] = (unsigned char)scale;
  }
}

template <typename T, int D, int BITS>
__device__ __forceinline__ void read_row(const CacheRowsArgs& a, const Place& p) {
  constexpr int PER = D / 8, CB = D * BITS / 8, SB = D / 32;
  const int t = threadIdx.x % PER;
  const unsigned char* base = a.cache + (max(p.page, 0LL) * a.c.H + p.h) * a.c.head_bytes();
  uint2 raw[2] = {};
  int scale[2] = {127, 127};  // (no such page: zeros)
  if (p.page >= 0) {
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const unsigned char* codes = base + (which * a.c.page_size + p.row) * (long long)CB + t * BITS;
      if constexpr (BITS == 4) raw[which].x = *reinterpret_cast<const unsigned*>(codes);
      else raw[which] = *reinterpret_cast<const uint2*>(codes);
      scale[which] = base[2LL * a.c.page_size * CB + ((long long)which * a.c.page_size + p.row) * SB + t / 4];
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float f = __uint_as_float((unsigned)scale[which] << 23);
    unsigned w[4];  // two bf16 each: exact, a code has at most four significant bits
    if constexpr (BITS == 4) {
      w[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[which].x, f, 0));
      w[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[which].x, f, 1));
      w[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[which].x, f, 2));
      w[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[which].x, f, 3));
    } else {
      w[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[which].x, f, false));
      w[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[which].x, f, true));
      w[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[which].y, f, false));
      w[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[which].y, f, true));
    }
    if (scale[which] == 255) w[0] = w[1] = w[2] = w[3] = 0x7fc07fc0u;
    unsigned char* dst = static_cast<unsigned char*>(which ? a.v : a.k);
    const Strides3& st = which ? a.sv : a.sk;
    T* row = reinterpret_cast<T*>(dst + p.b * st.batch + p.h * st.head + p.i * st.token) + 8 * t;
    if constexpr (std::is_same<T, float>::value) {
      reinterpret_cast<float4*>(row)[0] = bf16_pair(w[0], w[1]);
      reinterpret_cast<float4*>(row)[1] = bf16_pair(w[2], w[3]);
    } else {
      *reinterpret_cast<uint4*>(row) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}
template <typename T, int D, int BITS>
__global__ __launch_bounds__(256) void cache_read(CacheRowsArgs a) {
  Place p;
  if (place_of<D>(a, &p)) read_row<T, D, BITS>(a, p);
}
template <int D, int BITS>
__global__ __launch_bounds__(256) void cache_expand(CacheRowsArgs a, WindowShape w) {
  constexpr int PER = D / 8;
  Place p;
  p.i = blockIdx.x * (256 / PER) + threadIdx.x / PER, p.h = blockIdx.y, p.b = blockIdx.z;
  const WindowKeys keys = window_all_keys(w, window_seq_of(w, p.b));
  if (p.i >= min(keys.count, a.rows)) return;
  place_at(a, window_key(keys, p.i), &p);
  read_row<uint16_t, D, BITS>(a, p);
}

template <typename F>
hipError_t by_kind(const CacheRowsArgs& a, bool bf16, F f) {
  const int per = 256 / (a.c.d / 8);
  const dim3 grid((a.rows + per - 1) / per, a.c.H, a.c.B);
  auto with = [&](auto t, auto d) {
    if (a.c.bits == 4) f(t, d, std::integral_constant<int, 4>{}, grid);
    else f(t, d, std::integral_constant<int, 8>{}, grid);
  };
  auto sized = [&](auto t) {
    if (a.c.d == 128) with(t, std::integral_constant<int, 128>{});
    else with(t, std::integral_constant<int, 64>{});
  };
  if (bf16) sized(uint16_t{});
  else sized(float{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const CacheRowsArgs& a, bool bf16, hipStream_t st) {
  return by_kind(a, bf16, [&](auto t, auto d, auto bits, const dim3& grid) {
    cache_write<decltype(t), decltype(d)::value, decltype(bits)::value><<<grid, 256, 0, st>>>(a);
  });
}
hipError_t launch_cache_read(const CacheRowsArgs& a, bool bf16, hipStream_t st) {
  return by_kind(a, bf16, [&](auto t, auto d, auto bits, const dim3& grid) {
    cache_read<decltype(t), decltype(d)::value, decltype(bits)::value><<<grid, 256, 0, st>>>(a);
  });
}

hipError_t launch_cache_expand(const CacheRowsArgs& a, const WindowShape& w, hipStream_t st) {
  return by_kind(a, true, [&](auto t, auto d, auto bits, const dim3& grid) {
    if constexpr (std::is_same<decltype(t), uint16_t>::value) cache_expand<decltype(d)::value, decltype(bits)::value><<<grid, 256, 0, st>>>(a, w);
  });
}

}  // namespace usv
