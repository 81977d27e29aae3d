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
// Two at once (one v_cvt_pk_bf16_f32), the first in the low half.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// A byte offset past every buffer below, and raw buffers over a few rows of a
// tensor.  Loads past a buffer give zeros and stores past it are dropped, so tails
// of tokens and channels need no branch and no second address.
constexpr unsigned BUF_OOB = 0x80000000u;
struct RowsAt {  // walks a tensor's rows in steps
  const char* p;
  unsigned rb;  // bytes between rows; a step's rows span less than BUF_OOB
  __device__ __forceinline__ RowsAt(const void* t, long row0, long row_bytes)
      : p(static_cast<const char*>(t) + row0 * row_bytes), rb((unsigned)row_bytes) {}
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t rows(int n) const {
    return clip_rsrc(const_cast<char*>(p), (unsigned)n * rb);
  }
  __device__ __forceinline__ void step(int n) { p += (long)n * (int)rb; }
};

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
  // The same from a raw buffer at byte off; what lies past the buffer reads as
  // zeros, and so do channels from nv on (VEC: a lane without channels has an
  // offset past every buffer).
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, unsigned off, int nv) {
    if constexpr (VEC) {
      if constexpr (BYTES == 2) {
        r[0] = __builtin_amdgcn_raw_buffer_load_b16(rs, off, 0, 0);
      } else if constexpr (BYTES == 4) {
        r[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, 0);
      } else if constexpr (BYTES == 8) {
        const auto u = __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0);
        r[0] = u[0];
        r[1] = u[1];
      } else {
#pragma unroll
        for (int i = 0; i < NW / 4; ++i) {
          const auto u = __builtin_amdgcn_raw_buffer_load_b128(rs, off + 16 * i, 0, 0);
          r[4 * i] = u[0];
          r[4 * i + 1] = u[1];
          r[4 * i + 2] = u[2];
          r[4 * i + 3] = u[3];
        }
      }
    } else {
      auto at = [&](int i) { return i < nv ? off + i * (unsigned)sizeof(T) : BUF_OOB; };
      if constexpr (is_f32<T>::value) {
#pragma unroll
        for (int i = 0; i < C; ++i) r[i] = __builtin_amdgcn_raw_buffer_load_b32(rs, at(i), 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < NW; ++i) {
          const uint32_t lo = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, at(2 * i), 0, 0);
          const uint32_t hi = 2 * i + 1 < C ? (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, at(2 * i + 1), 0, 0) : 0;
          r[i] = lo | (hi << 16);
        }
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
      for (int i = 0; i < C / 2; ++i) u[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
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

// Stores the first nv of C channels at byte off of a raw buffer (see Piece::load).
template <typename T, int C, bool VEC>
__device__ __forceinline__ void store_piece(__amdgpu_buffer_rsrc_t rs, unsigned off, const float (&v)[C], int nv) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const unsigned at = i < nv ? off + i * (unsigned)sizeof(T) : BUF_OOB;
      if constexpr (is_f32<T>::value) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[i]), rs, at, 0, 0);
      else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)bf16_bits(v[i]), rs, at, 0, 0);
    }
  } else {
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
    typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
    constexpr int NW = (C * (int)sizeof(T) + 3) / 4;
    uint32_t u[NW];
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      if constexpr (is_f32<T>::value) u[i] = __float_as_uint(v[i]);
      else if constexpr (C == 1) u[i] = bf16_bits(v[0]);
      else u[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    }
    if constexpr (C * sizeof(T) == 2) {
      __builtin_amdgcn_raw_buffer_store_b16((uint16_t)u[0], rs, off, 0, 0);
    } else if constexpr (NW == 1) {
      __builtin_amdgcn_raw_buffer_store_b32(u[0], rs, off, 0, 0);
    } else if constexpr (NW == 2) {
      __builtin_amdgcn_raw_buffer_store_b64((u32x2_t{u[0], u[1]}), rs, off, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < NW / 4; ++i)
        __builtin_amdgcn_raw_buffer_store_b128((u32x4_t{u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]}), rs,
                                               off + 16 * i, 0, 0);
    }
  }
}

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// Logistic function (hardware 2^x and reciprocal, each within about an ulp; 1 +
// e^-x >= 1; x = -inf gives 0, +inf 1, NaN stays NaN).
__device__ __forceinline__ float sigmoid_acc(float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-LOG2E * x));
}
// log(1 + e^x) = max(x, 0) + log1p(e), e = e^-|x| in (0, 1], with
// log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3.  2 artanh(s) / s is a
// polynomial of degree 4 in s^2, fitted at Chebyshev points of [0, 1/9]
// (relative error 8e-9 as stored).  (log(1 + e) itself would lose the low bits of a
// small e, and steps of 0.001 are ordinary here.)
__device__ __forceinline__ float softplus_acc(float x) {
  const float e = __builtin_amdgcn_exp2f(-LOG2E * fabsf(x));
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
  float p = 0.28174657f;
  p = fmaf(p, q, 0.27961419f);
  p = fmaf(p, q, 0.40024854f);
  p = fmaf(p, q, 0.66666316f);
  p = fmaf(p, q, 2.0000000f);
  return fmaf(s, p, __builtin_elementwise_maximum(x, 0.f));  // (a NaN stays one)
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
