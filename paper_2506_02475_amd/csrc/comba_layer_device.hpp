// Device building blocks shared by the layer's operators (convolution,
// selective scan, group norm): pieces of consecutive channels, activations,
// sequence lookup and lane exchanges.
#pragma once

#include "comba_device.hpp"

namespace comba {

__device__ __forceinline__ void store_elem(float* p, float x) { *p = x; }
// The hardware conversion rounds to nearest even and keeps NaN a NaN.
__device__ __forceinline__ uint32_t bf16_bits(float x) {
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ __forceinline__ void store_elem(bf16_t* p, float x) { *p = (bf16_t)bf16_bits(x); }

// C consecutive channels as loaded.  VEC: one load of C * sizeof(T) bytes (the
// address is a multiple of that); else element by element, of which nv >= 1
// exist (the others repeat the last one).
template <typename T, int C, bool VEC>
struct Piece {
  static constexpr int BYTES = C * (int)sizeof(T), NW = (BYTES + 3) / 4;
  uint32_t r[NW];
  __device__ __forceinline__ void load(const T* p, int nv) {
    if constexpr (VEC) {
      if constexpr (BYTES == 2) {
        r[0] = *reinterpret_cast<const uint16_t*>(p);
      } else if constexpr (BYTES == 4) {
        r[0] = *reinterpret_cast<const uint32_t*>(p);
      } else if constexpr (BYTES == 8) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        r[0] = u.x;
        r[1] = u.y;
      } else {
#pragma unroll
        for (int i = 0; i < NW / 4; ++i) {
          const uint4 u = reinterpret_cast<const uint4*>(p)[i];
          r[4 * i] = u.x;
          r[4 * i + 1] = u.y;
          r[4 * i + 2] = u.z;
          r[4 * i + 3] = u.w;
        }
      }
    } else if constexpr (is_f32<T>::value) {
#pragma unroll
      for (int i = 0; i < C; ++i) r[i] = __float_as_uint(p[min(i, nv - 1)]);
    } else {
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        const uint32_t lo = p[min(2 * i, nv - 1)];
        const uint32_t hi = 2 * i + 1 < C ? p[min(2 * i + 1, nv - 1)] : 0;
        r[i] = lo | (hi << 16);
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (is_f32<T>::value) return __uint_as_float(r[i]);
    return __uint_as_float((i & 1) ? r[i / 2] & 0xFFFF0000u : r[i / 2] << 16);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < NW; ++i) r[i] = 0u;
  }
};

// Stores the first nv of C channels (VEC: nv is C or 0).
template <typename T, int C, bool VEC>
__device__ __forceinline__ void store_piece(T* p, const float (&v)[C], int nv) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < C; ++i)
      if (i < nv) store_elem(p + i, v[i]);
  } else if (nv > 0) {
    if constexpr (is_f32<T>::value) {
      if constexpr (C == 1) {
        *p = v[0];
      } else if constexpr (C == 2) {
        *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
      } else {
#pragma unroll
        for (int i = 0; i < C / 4; ++i)
          reinterpret_cast<float4*>(p)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
      }
    } else if constexpr (C == 1) {
      store_elem(p, v[0]);
    } else {
      uint32_t u[C / 2];
#pragma unroll
      for (int i = 0; i < C / 2; ++i) u[i] = bf16_bits(v[2 * i]) | (bf16_bits(v[2 * i + 1]) << 16);
      if constexpr (C == 2) {
        *reinterpret_cast<uint32_t*>(p) = u[0];
      } else if constexpr (C == 4) {
        *reinterpret_cast<uint2*>(p) = make_uint2(u[0], u[1]);
      } else {
#pragma unroll
        for (int i = 0; i < C / 8; ++i)
          reinterpret_cast<uint4*>(p)[i] = make_uint4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
      }
    }
  }
}

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// e^x: the hardware's 2^y with the rounding error of y = x log2(e) put back
// (y's absolute error is a relative one of the result: 5e-7 at |x| = 8 without).
__device__ __forceinline__ float exp_acc(float x) {
  const float y = x * LOG2E;
  const float e = __builtin_amdgcn_exp2f(y);
  // infinite y (x = -inf, or past the range): nothing to put back
  const float r = fabsf(y) < 1e30f ? fmaf(x, LOG2E, -y) * LN2 : 0.f;
  return fmaf(e, r, e);
}
// Logistic function (hardware reciprocal, about 1 ulp; 1 + e^-x >= 1).
__device__ __forceinline__ float sigmoid_acc(float x) {
  return __builtin_amdgcn_rcpf(1.f + exp_acc(-x));
}
// log(1 + e^x) = max(x, 0) + log1p(e), e = e^-|x| in (0, 1], with
// log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3: the odd series to s^13, whose
// remainder is below 2e-8 of the value.  (log(1 + e) itself would lose the low
// bits of a small e, and steps of 0.001 are ordinary here.)
__device__ __forceinline__ float softplus_acc(float x) {
  const float e = exp_acc(-fabsf(x));
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
  float p = 1.f / 13.f;
  p = fmaf(p, q, 1.f / 11.f);
  p = fmaf(p, q, 1.f / 9.f);
  p = fmaf(p, q, 1.f / 7.f);
  p = fmaf(p, q, 1.f / 5.f);
  p = fmaf(p, q, 1.f / 3.f);
  p = fmaf(p, q, 1.f);
  return fmaf(2.f * s, p, x > 0.f ? x : 0.f);
}

// Tokens [a, b) of sequence s, inside [0, Ttot] whatever the offsets hold.
__device__ __forceinline__ void seq_range(const int32_t* __restrict__ cu, int s, int Tseq, int Ttot,
                                          int& a, int& b) {
  if (!cu) {
    a = s * Tseq;
    b = a + Tseq;
    return;
  }
  a = min(max(cu[s], 0), Ttot);
  b = min(max(cu[s + 1], a), Ttot);
}

// Sum of two values over the lane pairs that differ in bit BIT: a lane whose
// bit is clear gets a's sum, the other b's.  (Level 2 pairs lane l with l ^ 7:
// any pairing that flips the bit serves a reduction that goes on to the lower
// bits.)
template <int BIT>
__device__ __forceinline__ float xpair(float a, float b) {
  if constexpr (BIT == 5) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else if constexpr (BIT == 4) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else {
    constexpr int CTRL = BIT == 3 ? 0x128 : BIT == 2 ? 0x141 : BIT == 1 ? 0x4E : 0xB1;
    const bool up = lane_id() & (1 << BIT);
    const float give = up ? a : b, keep = up ? b : a;
    return keep + dpp_upd<CTRL>(0.f, give);
  }
}
// The same for one value: both lanes get the sum.
template <int BIT>
__device__ __forceinline__ float xsum(float a) {
  if constexpr (BIT >= 4) {
    return xpair<BIT>(a, a);
  } else {
    constexpr int CTRL = BIT == 3 ? 0x128 : BIT == 2 ? 0x141 : BIT == 1 ? 0x4E : 0xB1;
    return a + dpp_upd<CTRL>(0.f, a);
  }
}
// Sums V values over the lanes that differ in bits TOP..LOW, and spreads the
// results: at each level the lanes with the bit clear go on with the first half
// of the values, the others with the second (a single value is summed in all
// lanes).  Leaves max(1, V >> levels) values in v[0..].
template <int V, int TOP, int LOW>
__device__ __forceinline__ void spread_sum(float* v) {
  if constexpr (TOP >= LOW) {
    if constexpr (V >= 2) {
#pragma unroll
      for (int k = 0; k < V / 2; ++k) v[k] = xpair<TOP>(v[k], v[k + V / 2]);
      spread_sum<V / 2, TOP - 1, LOW>(v);
    } else {
      v[0] = xsum<TOP>(v[0]);
      spread_sum<1, TOP - 1, LOW>(v);
    }
  }
}

}  // namespace comba
