// Linear attention with a decay for each head, in chunks of 64 tokens.  Per head,
// with G_r the sum of a chunk's log-decays up to row r and S the state entering it:
//
//   o_r   = scale (sum_{j <= r} e^{G_r - G_j} (q_r . k_j) v_j + e^{G_r} S^T q_r)
//   S'    = e^{G_end} S + sum_j e^{G_end - G_j} k_j v_j^T
//   dS    = e^{G_end} dS' + scale sum_r e^{G_r} q_r do_r^T        (dS' of the next chunk)
//   dq_r  = scale (sum_{j <= r} e^{G_r - G_j} (do_r . v_j) k_j + e^{G_r} S do_r)
//   dk_j  = scale sum_{r >= j} e^{G_r - G_j} (do_r . v_j) q_r + e^{G_end - G_j} dS' v_j
//   dv_j  = scale sum_{r >= j} e^{G_r - G_j} (q_r . k_j) do_r + e^{G_end - G_j} dS'^T k_j
//   dg_t  = the sum over all pairs j < t <= r of a pair's weight times its products:
//           both tokens in the chunk, one of them, or none (e^{G_end} <dS', S>).
//
// G is summed in 64 bits.  A row's weights towards its chunk's ends are formed from those
// sums; a pair's from two sums rounded to fp32 (bf16) or to two floats each (fp32): see Sums.
// Masked pairs' weights are formed as well (Inf where a decay is strong) and then dropped by
// a select, which takes nothing from what it drops.
// bf16 operands of the matrix products are rounded: the pairs' weighted products (o, dq, dk,
// dv), an entering state (o, dq; by way of its fp16) and a leaving one's gradient (dk, dv).  With
// the result's own rounding that is 2.4e-3 of a tensor's 2-norm, where one rounding is 1.7e-3;
// two terms of every operand would double the matrix instructions and the kept states.
#include "comba_block_launch.h"
#include "comba_layer_device.hpp"

namespace comba {

// ---- matrix products -----------------------------------------------------------
// Eight values of an operand along the summed index; bf16 on the bf16 matrix
// instruction, fp32 on the fp32 one (eight of its steps of one value a lane).
template <typename T> struct Frag;
template <> struct Frag<bf16_t> {
  bf16x8 x;
};
template <> struct Frag<float> {
  float x[8];
};
__device__ __forceinline__ floatx4 mma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.x, b.x, c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mma(const Frag<float>& a, const Frag<float>& b, floatx4 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[e], b.x[e], c, 0, 0, 0);
  return c;
}
template <typename T, bool VEC>
__device__ __forceinline__ Frag<T> as_frag(const Piece<T, 8, VEC>& p) {
  Frag<T> f;
  if constexpr (is_f32<T>::value) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.x[e] = __uint_as_float(p.r[e]);
  } else {
    f.x = __builtin_bit_cast(bf16x8, make_uint4(p.r[0], p.r[1], p.r[2], p.r[3]));
  }
  return f;
}
// Two accumulators as an operand: the lane's rows 4 (l / 16) .. + 3 of both.
template <typename T>
__device__ __forceinline__ Frag<T> frag_of(const floatx4& a, const floatx4& b) {
  Frag<T> f;
  if constexpr (is_f32<T>::value) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f.x[e] = a[e], f.x[4 + e] = b[e];
  } else {
    f.x = __builtin_bit_cast(bf16x8, make_uint4(bf16_pair(a[0], a[1]), bf16_pair(a[2], a[3]),
                                                bf16_pair(b[0], b[1]), bf16_pair(b[2], b[3])));
  }
  return f;
}
// Element offset in a tile of rows of LD bf16 (a multiple of 64; fp32: twice the bytes),
// whose pieces of eight are exchanged inside a row so that, bf16 and lanes taken in order,
// what these accesses touch at once falls on distinct ones of the 64 banks: 16 rows of one
// piece (ld_row, st_pairs), rows r .. r + 3 and r + 8 .. r + 11 of two pieces (ld_col), whole
// rows (st_row8), four rows of four (weighted values on their way in).  ld_col_acc does not
// have it: its rows r .. r + 3 and r + 4 .. r + 7 are exchanged by one bit only, so two rows
// share their banks.  Counted, conflict cycles of LDS's busy ones: scans (ld_col) 0, outputs
// 44% at heads of 128 and 47% at 256, gradients 34%, more than ld_col_acc alone explains.
template <int LD>
__device__ __forceinline__ int swz(int row, int col) {
  const int x = LD == 64 ? ((row & 2) << 1) | ((row >> 2) & 2) | ((row >> 2) & 1)
                         : ((row & 3) << 2) | ((row >> 2) & 2) | ((row >> 2) & 1);
  return row * LD + ((((col >> 3) ^ x) << 3) | (col & 7));
}
// The lane's number as a value of its own: tile addresses formed from it stay where they
// are used (the compiler would keep those of every tile in registers across a loop).
__device__ __forceinline__ int fresh_lane() {
  int l = lane_id();
  asm volatile("" : "+v"(l));
  return l;
}
// From such a tile:
// eight consecutive elements of row (lane % 16), from column col + 8 (lane / 16).
template <int LD, typename T>
__device__ __forceinline__ Frag<T> ld_row(const T* tile, int row, int col, int lane = lane_id()) {
  const T* p = tile + swz<LD>(row + (lane & 15), col + 8 * (lane >> 4));
  Frag<T> f;
  if constexpr (is_f32<T>::value) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    f.x[0] = a.x, f.x[1] = a.y, f.x[2] = a.z, f.x[3] = a.w;
    f.x[4] = b.x, f.x[5] = b.y, f.x[6] = b.z, f.x[7] = b.w;
  } else {
    f.x = *reinterpret_cast<const bf16x8*>(p);
  }
  return f;
}
// Column col + lane % 16 at rows r0 .. r0 + 3 and r1 .. r1 + 3.
template <int LD, typename T>
__device__ __forceinline__ Frag<T> ld_col2(const T* tile, int r0, int r1, int col, int lane) {
  const int s = lane & 15;
  Frag<T> f;
  if constexpr (is_f32<T>::value) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f.x[e] = tile[swz<LD>(r0 + e, col + s)];
      f.x[4 + e] = tile[swz<LD>(r1 + e, col + s)];
    }
  } else {
    const int at = s >> 2, c = col + 4 * (s & 3);
    f.x = ld_tr8(tile, TrOff{swz<LD>(r0 + at, c), swz<LD>(r1 + at, c)});
  }
  return f;
}
// The same at rows r0 + 8 (lane / 16) .. + 7 ...
template <int LD, typename T>
__device__ __forceinline__ Frag<T> ld_col(const T* tile, int r0, int col, int lane = lane_id()) {
  const int r = r0 + 8 * (lane >> 4);
  return ld_col2<LD>(tile, r, r + 4, col, lane);
}
// ... and in the row order of frag_of: 4 (lane / 16) .. + 3 of two blocks of 16.
template <int LD, typename T>
__device__ __forceinline__ Frag<T> ld_col_acc(const T* tile, int r0, int col, int lane = lane_id()) {
  const int r = r0 + 4 * (lane >> 4);
  return ld_col2<LD>(tile, r, r + 16, col, lane);
}
template <int LD, typename T, bool VEC>
__device__ __forceinline__ void st_row8(T* tile, int row, int col, const Piece<T, 8, VEC>& p) {
  uint4* d = reinterpret_cast<uint4*>(tile + swz<LD>(row, col));
  d[0] = make_uint4(p.r[0], p.r[1], p.r[2], p.r[3]);
  if constexpr (is_f32<T>::value) d[1] = make_uint4(p.r[4], p.r[5], p.r[6], p.r[7]);
}
// Four values at columns col .. col + 3 (a multiple of four).
template <int LD, typename T>
__device__ __forceinline__ void st_row4(T* tile, int row, int col, const floatx4& x) {
  T* d = tile + swz<LD>(row, col);
  if constexpr (is_f32<T>::value) *reinterpret_cast<float4*>(d) = make_float4(x[0], x[1], x[2], x[3]);
  else *reinterpret_cast<uint2*>(d) = make_uint2(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]));
}

// ---- chunks and rows --------------------------------------------------------------
// n tokens' rows of one head as a raw buffer: what lies behind the last row reads as
// zeros, and stores there are dropped.
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t head_rows(const void* t, long tok, long row, long col, int n, int d) {
  const T* p = static_cast<const T*>(t) + tok * row + col;
  const unsigned bytes = n > 0 ? (unsigned)(((long)(n - 1) * row + d) * (long)sizeof(T)) : 0u;
  return clip_rsrc(const_cast<T*>(p), bytes);
}
// Columns col .. col + C - 1 of row r; columns from d on are zeros.
template <typename T, int C, bool VEC>
__device__ __forceinline__ void load_piece(Piece<T, C, VEC>& p, __amdgpu_buffer_rsrc_t rs, int r, unsigned row_bytes,
                                           int col, int d) {
  const unsigned off = (unsigned)r * row_bytes + (unsigned)col * (unsigned)sizeof(T);
  if constexpr (VEC) p.load(rs, col < d ? off : BUF_OOB, C);
  else p.load(rs, off, d - col);
}
template <typename T, bool VEC>
__device__ __forceinline__ void load8(Piece<T, 8, VEC>& p, __amdgpu_buffer_rsrc_t rs, int r, unsigned row_bytes, int col,
                                      int d) {
  load_piece<T, 8, VEC>(p, rs, r, row_bytes, col, d);
}
template <typename T, bool VEC>
__device__ __forceinline__ Frag<T> load_frag(__amdgpu_buffer_rsrc_t rs, int row, unsigned row_bytes, int col, int d) {
  Piece<T, 8, VEC> p;
  load8(p, rs, row + (lane_id() & 15), row_bytes, col + 8 * (lane_id() >> 4), d);
  return as_frag<T, VEC>(p);
}
template <typename T, bool VEC>
__device__ __forceinline__ void store4c(__amdgpu_buffer_rsrc_t rs, int r, unsigned row_bytes, int col, int d,
                                        const floatx4& x) {
  const float v[4] = {x[0], x[1], x[2], x[3]};
  const unsigned off = (unsigned)r * row_bytes + (unsigned)col * (unsigned)sizeof(T);
  store_piece<T, 4, VEC>(rs, col < d ? off : BUF_OOB, v, d - col);
}

// The piece of a slot: sequence, its first token and length, the piece's number.  A
// sequence's slots start at start / unit + its number (fixed rows: at its number times
// `per`).  Offsets are clamped into the tokens whatever they hold.
struct Slot {
  int seq, piece, t0, len;
};
__device__ __forceinline__ Slot find_slot(const DecayArgs& a, int slot, int unit) {
  Slot s;
  if (!a.cu_seqlens) {
    const int per = max((a.Tseq + unit - 1) / unit, 1);
    s.seq = slot / per;
    s.piece = slot % per;
  } else {
    int lo = 0, hi = a.S;  // the last sequence whose slots start at or before this one
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (min(max(a.cu_seqlens[mid], 0), a.Ttot) / unit + mid <= slot) lo = mid;
      else hi = mid;
    }
    s.seq = lo;
    s.piece = max(slot - (min(max(a.cu_seqlens[lo], 0), a.Ttot) / unit + lo), 0);
  }
  int b;
  seq_range(a.cu_seqlens, s.seq, a.Tseq, a.Ttot, s.t0, b);
  s.len = b - s.t0;
  return s;
}
__device__ __forceinline__ int first_slot(const DecayArgs& a, const Slot& s, int unit) {
  return a.cu_seqlens ? s.t0 / unit + s.seq : s.seq * max((a.Tseq + unit - 1) / unit, 1);
}

// A token's log-decay, and the sums over a chunk (lane = row, 64 bits, base 2).
__device__ __forceinline__ float gate_of(const DecayArgs& a, long tok, int h) {
  if (a.g_head) return static_cast<const float*>(a.g)[h];
  const long at = tok * a.g_row + h;
  return a.g_f32 ? static_cast<const float*>(a.g)[at] : bf2f(static_cast<const bf16_t*>(a.g)[at]);
}
// The same of n tokens from tok on, one a lane, zeros behind them.  As two halves from a
// raw buffer (bf16: the lower one from behind it), so that no load stands under a branch
// and what is in flight is first touched where it is used.  Per head: `head`.
struct Gates {
  uint32_t lo, hi;
  int n;
  __device__ __forceinline__ void load(const DecayArgs& a, long tok, int h, int count) {
    n = count;
    const unsigned e = a.g_f32 ? 4 : 2, off = (unsigned)lane_id() * (unsigned)a.g_row * e;
    const char* p = static_cast<const char*>(a.g) + (tok * a.g_row + h) * e;
    const auto rs = clip_rsrc(const_cast<char*>(p), count > 0 && !a.g_head ? (unsigned)((count - 1) * (int)a.g_row + 1) * e : 0u);
    hi = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, off + (e - 2), 0, 0);
    lo = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, a.g_f32 ? off : BUF_OOB, 0, 0);
  }
  __device__ __forceinline__ float get(float head) const {
    const float x = __uint_as_float(hi << 16 | lo);
    return lane_id() < n ? x + head : 0.f;  // (per head x is zero, else head is)
  }
};
template <int CTRL, int ROWMASK = 0xF>
__device__ __forceinline__ double dpp_add(double x) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  const i32x2 u = __builtin_bit_cast(i32x2, x);
  const i32x2 y = {__builtin_amdgcn_update_dpp(0, u[0], CTRL, ROWMASK, 0xF, false),
                   __builtin_amdgcn_update_dpp(0, u[1], CTRL, ROWMASK, 0xF, false)};
  return x + __builtin_bit_cast(double, y);
}
__device__ __forceinline__ double read_lane(double x, int lane) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  const i32x2 u = __builtin_bit_cast(i32x2, x);
  return __builtin_bit_cast(double, i32x2{__builtin_amdgcn_readlane(u[0], lane), __builtin_amdgcn_readlane(u[1], lane)});
}
__device__ __forceinline__ double gate_sum(float g) {
  g = g < -128.f ? -128.f : g;
  double x = (double)g * 1.4426950408889634074;
  x = dpp_add<0x111>(x);  // as wave_prefix_sum
  x = dpp_add<0x112>(x);
  x = dpp_add<0x114>(x);
  x = dpp_add<0x118>(x);
  x = dpp_add<0x142, 0xA>(x);
  return dpp_add<0x143, 0xC>(x);
}
// Pair weights from a chunk's sums.  BOTH (fp32): of two floats each, so that a difference
// is within two roundings of itself.  Else (bf16) of one: sums are below 2^14 (64 rows of 128 log2(e) at
// most) and there within 2^-11, a difference within 2^-10 and a weight within ln(2) 2^-10 =
// 7e-4, a sixth of the half step (2^-8) that its product is rounded by next; of sums below
// 2^7, the ordinary ones, 5e-6.
struct Sums {
  float hi[DC_CH], lo[DC_CH];
  // 2^(G - G_j) of four j from j0 on
  template <bool BOTH>
  __device__ __forceinline__ floatx4 weights(float gh, float gl, int j0) const {
    const floatx4 h = *reinterpret_cast<const floatx4*>(hi + j0);
    floatx4 d;
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = gh - h[e];
    if constexpr (BOTH) {
      const floatx4 l = *reinterpret_cast<const floatx4*>(lo + j0);
#pragma unroll
      for (int e = 0; e < 4; ++e) d[e] += gl - l[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = __builtin_amdgcn_exp2f(d[e]);
    return d;
  }
};

// fp32 as the sum of three bf16: products with an exact bf16 operand keep 24 bits.
__device__ __forceinline__ void split3(float x, float y, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  uint32_t rest;
  split2(x, y, hi, rest);
  const float ax = x - __uint_as_float(hi << 16), ay = y - __uint_as_float(hi & 0xFFFF0000u);
  split2(ax, ay, mid, lo);
}

// ---- kept states -------------------------------------------------------------------
// A state [dv][dk] lies in blocks of 16 rows and CB columns, a block in the order in which
// a wave's lanes hold it, 16 bytes a lane: lane p has row p % 16 and the p / 16-th piece of
// the block's columns (bf16, 32 columns: in row8_col's order).  A wave so writes whole
// lines; rows and columns behind the heads' sizes are kept too, as the zeros they are.
// bf16: the entering states are kept as fp16 with one power-of-two scale a block (the scales
// behind the blocks), the gradients as bf16.  The products take both rounded to bf16, but
// dg's part from both directions, <dS', S>, takes S as kept: a rounding of S to bf16
// alone would put dg's error at 1.4 roundings, fp16's (an eighth, down to 2^-29 of a
// block's largest) vanishes beside dg's own.
// Four values by 1 / scale as fp16, and back; the scale takes a block's largest, m, to
// [2^14, 2^15), and is NaN where m is not finite.
__device__ __forceinline__ float half_inv_scale(float m) { return __int_as_float((142 - q_exponent(m)) << 23); }
__device__ __forceinline__ uint2 pack_half4(const floatx4& x, float inv) {
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  const f16x4 h = {(_Float16)(x[0] * inv), (_Float16)(x[1] * inv), (_Float16)(x[2] * inv), (_Float16)(x[3] * inv)};
  return __builtin_bit_cast(uint2, h);
}
__device__ __forceinline__ float4 unpack_half4(uint2 u, float s) {
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  const f16x4 h = __builtin_bit_cast(f16x4, u);
  return make_float4((float)h[0] * s, (float)h[1] * s, (float)h[2] * s, (float)h[3] * s);
}
template <typename T, int DK>
struct StateLayout {
  static constexpr int CB = is_f32<T>::value || DK == 64 ? 16 : 32;
  static constexpr int E = 16 / (int)sizeof(T);  // values of a lane
  static constexpr int PB = 16 * CB / E;         // pieces of a block
  int blocks;           // side by side
  unsigned data, bytes; // the blocks', with their scales
  __device__ __forceinline__ StateLayout(int dk, int dv)
      : blocks((dk + CB - 1) / CB), data((unsigned)(((dv + 15) & ~15) * blocks * CB) * (unsigned)sizeof(T)),
        bytes((unsigned)state_bytes(!is_f32<T>::value, dk, dv)) {}
  // byte offset of a block's scale
  __device__ __forceinline__ unsigned scale_at(int vblk, int cblk) const {
    const unsigned b = (unsigned)(vblk * blocks + cblk);
    return cblk < blocks && b * (PB * 16u) < data ? data + b * 4u : BUF_OOB;
  }
  // byte offset of a block's piece p; what lies outside the state is behind its bytes
  __device__ __forceinline__ unsigned at(int vblk, int cblk, int p) const {
    const unsigned off = (unsigned)((vblk * blocks + cblk) * PB + p) * 16u;
    return cblk < blocks && off < data ? off : BUF_OOB;
  }
  static __device__ __forceinline__ int col_of(int p) {  // first column of piece p in its block
    const int g = p >> 4;
    return E * (CB == 32 && E == 8 ? ((g & 1) << 1) | (g >> 1) : g);
  }
};
// A tile of 64 rows (value columns) and COLS key columns of a kept state, through registers
// into LDS (ENTERS: an entering state, as fp16).
template <typename T, int DK, int COLS, bool ENTERS>
struct StateTile {
  typedef StateLayout<T, DK> L;
  static constexpr bool Q = ENTERS && !is_f32<T>::value;
  static constexpr int N = 64 * COLS / L::E / 256;
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  u32x4_t r[N];
  float scale[Q ? N : 1];
  static __device__ __forceinline__ void where(int i, int& vblk, int& cblk, int& p) {
    const int idx = threadIdx.x + 256 * i, b = idx / L::PB;
    p = idx % L::PB;
    vblk = b / (COLS / L::CB);
    cblk = b % (COLS / L::CB);
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, const L& l, int v0, int c0) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int vblk, cblk, p;
      where(i, vblk, cblk, p);
      vblk += v0 / 16;
      cblk += c0 / L::CB;
      r[i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, l.at(vblk, cblk, p), 0, 0));
      if constexpr (Q)
        scale[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, l.scale_at(vblk, cblk), 0, 0));
    }
  }
  __device__ __forceinline__ void store(T* tile) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int vblk, cblk, p;
      where(i, vblk, cblk, p);
      u32x4_t x = r[i];
      if constexpr (Q) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float4 y = unpack_half4(make_uint2(x[2 * e], x[2 * e + 1]), scale[i]);
          x[2 * e] = bf16_pair(y.x, y.y);
          x[2 * e + 1] = bf16_pair(y.z, y.w);
        }
      }
      *reinterpret_cast<u32x4_t*>(tile + swz<COLS>(16 * vblk + (p & 15), L::CB * cblk + L::col_of(p))) = x;
    }
  }
};
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t state_rsrc(const void* kept, long slot_head, unsigned bytes) {
  return clip_rsrc(const_cast<char*>(static_cast<const char*>(kept)) + slot_head * (long)bytes, bytes);
}

// ---- the scans ---------------------------------------------------------------------
// A workgroup walks the chunks of one segment of one sequence and head, holds DC_BV value
// columns of the state in fp32 accumulators (wave w: key rows (w % 4) DK / 4 .., columns
// 16 (w / 4) ..), and keeps what it holds before each chunk.  Forward: keys k, values v,
// weights e^{G_end - G_j}.  REV, for the states' gradients, from the last chunk to the
// first: keys q, values do, weights scale e^{G_r}.  LOCAL: a segment's end from a zero
// state, for the segments behind it.  The weights multiply the value columns, of which a workgroup has few, and there
// fp32 becomes three bf16 against the keys as they are: the state's sums keep 24 bits.
//
// Bound by the latency of a chunk's chain (its decays, the weighted values into LDS, their
// products), not by what it moves: so two tiles in LDS, the next chunk being staged while
// one is multiplied, one barrier a chunk, and loads two chunks ahead of their staging.
// 4 x 4,096 tokens, 16 heads of 128, bf16: forward 84 us (77 at best), 268 MB, 3.2 TB/s; REV
// 101 (93), 403 MB, 4.0 TB/s; no LDS bank conflicts.  A row of 15,777 tokens: 1.1 us a chunk.
constexpr int SCAN_THREADS = 512;
// Keys; weighted values (bf16: three terms, fp32: both tiles' side by side).
template <typename T, int DK>
struct ScanTiles {
  static constexpr bool F32 = is_f32<T>::value;
  static constexpr int VLD = F32 ? 64 : 128;
  T key[2][DC_CH * DK], val[F32 ? 1 : 2][DC_CH * VLD];
  float wts[2][DC_CH], fades[4];  // of chunk c: the rows' weights [c % 2], its decay [c % 4]
  __device__ __forceinline__ T* v(int b) { return val[F32 ? 0 : b]; }
  static __device__ __forceinline__ int col(int b) { return F32 ? 32 * b : 0; }
};

template <typename T, int DK, bool REV, bool LOCAL, bool VEC>
__global__ __launch_bounds__(SCAN_THREADS) void k_decay_scan(DecayArgs a, int units) {
  constexpr bool F32 = is_f32<T>::value;
  constexpr int VLD = ScanTiles<T, DK>::VLD, NT = F32 ? 1 : 3;
  constexpr int MT = DK / 64;
  __shared__ __align__(16) ScanTiles<T, DK> t;

  // the splits of one head's state on one XCD (they read the same keys), heads dealt
  // over the XCDs
  const int NS = (a.dv + DC_BV - 1) / DC_BV;
  const int id = blockIdx.x % (8 * NS), u = blockIdx.x / (8 * NS) * 8 + id % 8, split = id / 8;
  if (u >= units) return;
  const int slot = u / a.H, h = u % a.H, j0 = split * DC_BV;
  const Slot sq = find_slot(a, slot, a.seglen);
  const int first = sq.piece * a.seglen;
  if (sq.piece > 0 && first >= sq.len) return;
  const int n = min(a.seglen, sq.len - first), nc = (n + DC_CH - 1) / DC_CH;
  const int base = first_slot(a, sq, a.seglen);
  const int segs = max((sq.len + a.seglen - 1) / a.seglen, 1);
  if (LOCAL && sq.piece == (REV ? 0 : segs - 1)) return;  // no segment comes after it
  const int wave = wave_id_s(), w = wave & 3, lane = lane_id(), r16 = lane & 15, g4 = lane >> 4;
  const int c0 = 16 * (wave >> 2);  // of the workgroup's columns

  const int hx = REV ? h / (a.H / a.Hq) : h / (a.H / a.Hk), hv = REV ? h : h / (a.H / a.Hv);
  const long xrow = REV ? a.q_row : a.k_row, yrow = REV ? (long)a.H * a.dv : a.v_row;
  const void *X = REV ? a.q : a.k, *Y = REV ? a.dO : a.v;
  const long tok0 = (long)sq.t0 + first;

  // ---- a chunk's inputs
  struct Inputs {
    Piece<T, 8, VEC> k[MT];
    Piece<T, 4, VEC> v;
  } in0, in1;
  Gates g0, g1;
  const float ghead = a.g_head ? static_cast<const float*>(a.g)[h] : 0.f;
  auto tokens = [&](int it, long& tok) {  // of the it-th chunk of the walk (behind the last one: none)
    const int c = REV ? nc - 1 - it : it;
    tok = tok0 + (long)c * DC_CH;
    return it < nc ? min(DC_CH, n - c * DC_CH) : 0;
  };
  auto load_gates = [&](Gates& g, int it) {  // (wave 0's: the others' lie behind the buffer)
    long tok;
    const int m = tokens(it, tok);
    g.load(a, tok, h, wave == 0 ? m : 0);
  };
  auto load = [&](Inputs& in, int it) {
    long tok;
    const int m = tokens(it, tok);
    const auto rx = head_rows<T>(X, tok, xrow, (long)hx * a.dk, m, a.dk);
    const auto ry = head_rows<T>(Y, tok, yrow, (long)hv * a.dv, m, a.dv);
    load_piece(in.v, ry, threadIdx.x / 8, (unsigned)yrow * sizeof(T), j0 + threadIdx.x % 8 * 4, a.dv);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int idx = threadIdx.x + i * SCAN_THREADS;
      load8(in.k[i], rx, idx / (DK / 8), (unsigned)xrow * sizeof(T), idx % (DK / 8) * 8, a.dk);
    }
  };
  load_gates(g0, 0);
  load_gates(g1, 1);
  load(in0, 0);
  load(in1, 1);

  // ---- the state that enters
  floatx4 S[MT];
  const int row0 = w * (DK / 4) + 4 * g4, scol = j0 + c0 + r16;  // key rows row0 + 16 m + i, value column
  auto each = [&](auto fn) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) S[m][i] = fn(S[m][i], row0 + 16 * m + i, scol);
  };
  const long ends = (long)NS * DC_BV * DK;  // floats of a segment's end
  auto end_at = [&](int sl) {
    return a.segS + ((long)sl * a.H + h) * ends + (((long)split * 8 + wave) * 64 + lane) * (MT * 4);
  };
  const float* entering = REV ? a.dht : a.h0;
  const long sbase = ((long)sq.seq * a.H + h) * a.dk * a.dv;
  {
    const int before = LOCAL ? 0 : REV ? segs - 1 - sq.piece : sq.piece;  // segments it has behind it
    auto nth = [&](int p) { return base + (REV ? sq.piece + 1 + p : sq.piece - 1 - p); };  // the nearest first
    double f = 0.;
    for (int p = 0; p < before; ++p) f += a.segG[(long)nth(p) * a.H + h];
    const float far = __builtin_amdgcn_exp2f((float)f);
    each([&](float, int r, int c) {
      return !LOCAL && entering && r < a.dk && c < a.dv ? far * entering[sbase + (long)r * a.dv + c] : 0.f;
    });
    double between = 0.;
    for (int p = 0; p < before; ++p) {
      const int sl = nth(p);
      const float f2 = __builtin_amdgcn_exp2f((float)between);
      const float4* e = reinterpret_cast<const float4*>(end_at(sl));
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const float4 x = e[m];
        S[m][0] = fmaf(f2, x.x, S[m][0]);
        S[m][1] = fmaf(f2, x.y, S[m][1]);
        S[m][2] = fmaf(f2, x.z, S[m][2]);
        S[m][3] = fmaf(f2, x.w, S[m][3]);
      }
      between += a.segG[(long)sl * a.H + h];
    }
  }

  // A chunk's decay and its rows' weights, by wave 0, a step before they are used
  double total = 0.;
  auto weigh = [&](const Gates& g, int it) {
    if (wave != 0) return;
    const double G = gate_sum(g.get(ghead)), Gend = read_lane(G, 63);
    total += Gend;
    t.wts[it & 1][lane] = REV ? a.scale * __builtin_amdgcn_exp2f((float)G) : __builtin_amdgcn_exp2f((float)(Gend - G));
    if (lane == 0) t.fades[it & 3] = __builtin_amdgcn_exp2f((float)Gend);
  };
  auto stage = [&](int b, const Inputs& in, int it) {  // into tile b
    const float f = t.wts[it & 1][threadIdx.x / 8];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int idx = threadIdx.x + i * SCAN_THREADS;
      st_row8<DK>(t.key[b], idx / (DK / 8), idx % (DK / 8) * 8, in.k[i]);
    }
    const int row = threadIdx.x / 8, col = threadIdx.x % 8 * 4 + t.col(b);
    const float x[4] = {f * in.v.get(0), f * in.v.get(1), f * in.v.get(2), f * in.v.get(3)};
    if constexpr (F32) {
      st_row4<VLD>(t.v(b), row, col, floatx4{x[0], x[1], x[2], x[3]});
    } else {
      uint2 y[3];
      split3(x[0], x[1], y[0].x, y[1].x, y[2].x);
      split3(x[2], x[3], y[0].y, y[1].y, y[2].y);
#pragma unroll
      for (int e = 0; e < 3; ++e) *reinterpret_cast<uint2*>(t.v(b) + swz<VLD>(row, 32 * e + col)) = y[e];
    }
  };
  // The state before a chunk: a lane has four key rows of a value column (bf16: exchanged to
  // eight in a row).  No store stands under a branch: what waits for the loads behind it
  // counts the memory operations in between, and would count too few.
  const StateLayout<T, DK> layout(a.dk, a.dv);
  const int kslot = first_slot(a, sq, DC_CH) + first / DC_CH;
  const int vblk = (j0 + c0) / 16;
  auto keep = [&](int it) {
    const int c = REV ? nc - 1 - it : it;
    const auto rs = state_rsrc<T>(REV ? a.dkept : a.kept, (long)(kslot + c) * a.H + h, layout.bytes);
    typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
    auto put = [&](int cblk, int p, uint4 y) {
      __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{y.x, y.y, y.z, y.w}, rs, layout.at(vblk, cblk, p), 0, 0);
    };
    // four values as bf16; forward: as fp16 by the block's scale, which one lane stores
    auto pack = [&](const floatx4& x, float inv) {
      return REV ? make_uint2(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])) : pack_half4(x, inv);
    };
    auto scaled = [&](float most, int cblk) {
      most = rowgroup_max(max16(most));
      __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(q_scale(most)), rs,
                                            lane == 0 ? layout.scale_at(vblk, cblk) : BUF_OOB, 0, 0);
      return half_inv_scale(most);
    };
    if constexpr (F32) {
#pragma unroll
      for (int m = 0; m < MT; ++m) put(w * MT + m, lane, __builtin_bit_cast(uint4, S[m]));
    } else if constexpr (MT == 1) {
      const uint2 x = pack(S[0], REV ? 0.f : scaled(nmax_abs4(0.f, S[0]), w));
      const auto u = __builtin_amdgcn_permlane16_swap(x.x, x.x, false, false);
      const auto v = __builtin_amdgcn_permlane16_swap(x.y, x.y, false, false);
      // (both lanes of a pair have the eight: the odd ones store behind the state)
      put(g4 & 1 ? layout.blocks : w, r16 + 16 * (g4 >> 1), make_uint4(u[0], v[0], u[1], v[1]));
    } else {
#pragma unroll
      for (int m = 0; m < MT; m += 2) {
        const int cblk = w * (MT / 2) + m / 2;
        const float inv = REV ? 0.f : scaled(nmax_abs4(nmax_abs4(0.f, S[m]), S[m + 1]), cblk);
        put(cblk, lane, row8_from_pieces(pack(S[m], inv), pack(S[m + 1], inv)));
      }
    }
  };
  // REV, for dg: the products of the gradient that leaves a chunk (in fp32 here: of two states
  // rounded to bf16 dg would have another half of a rounding's error) with the state that
  // enters it, a partial sum for each wave.
  struct Entering {
    uint32_t r[MT][F32 ? 4 : 2];
    float scale[F32 ? 1 : (MT + 1) / 2];
  } e0, e1;
  auto load_state = [&](Entering& e, int it) {
    const int c = REV ? nc - 1 - it : it;
    const bool on = it < nc && a.dg;
    const auto rs = state_rsrc<T>(a.kept, (long)(kslot + c) * a.H + h, layout.bytes);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      // (the lane's four key rows: as keep() left them)
      if constexpr (F32) {
        const auto u = __builtin_amdgcn_raw_buffer_load_b128(rs, on ? layout.at(vblk, w * MT + m, lane) : BUF_OOB, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) e.r[m][i] = u[i];
      } else {
        const int o = MT == 1 ? g4 >> 1 : 2 * (m & 1) + (g4 >> 1), piece = MT == 1 ? o : ((o & 1) << 1) | (o >> 1);
        const unsigned at = layout.at(vblk, MT == 1 ? w : w * (MT / 2) + m / 2, r16 + 16 * piece) + 8 * (g4 & 1);
        const auto u = __builtin_amdgcn_raw_buffer_load_b64(rs, on ? at : BUF_OOB, 0, 0);
        e.r[m][0] = u[0];
        e.r[m][1] = u[1];
        if (m % 2 == 0) {
          const unsigned sc = layout.scale_at(vblk, MT == 1 ? w : w * (MT / 2) + m / 2);
          e.scale[m / 2] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, on ? sc : BUF_OOB, 0, 0));
        }
      }
    }
  };
  auto meet = [&](const Entering& e, int it) {
    float s = 0.f;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float4 x;
      if constexpr (F32) x = __builtin_bit_cast(float4, make_uint4(e.r[m][0], e.r[m][1], e.r[m][2], e.r[m][3]));
      else x = unpack_half4(make_uint2(e.r[m][0], e.r[m][1]), e.scale[m / 2]);
      s = fmaf(S[m][0], x.x, fmaf(S[m][1], x.y, fmaf(S[m][2], x.z, fmaf(S[m][3], x.w, s))));
    }
    s = wave_sum(s);
    const long at = ((long)(kslot + nc - 1 - it) * a.H + h) * NS * 8;
    const auto rs = clip_rsrc(a.met + at, a.dg ? (unsigned)NS * 32u : 0u);
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(s), rs, lane == 0 ? (unsigned)(split * 8 + wave) * 4u : BUF_OOB, 0, 0);
  };
  if constexpr (REV && !LOCAL) {
    load_state(e0, 0);
    load_state(e1, 1);
  }
  weigh(g0, 0);
  weigh(g1, 1);
  load_gates(g0, 2);
  load_gates(g1, 3);
  __syncthreads();
  stage(0, in0, 0);
  load(in0, 2);
  __syncthreads();
  auto step = [&](int b, Inputs& in, Gates& g, Entering& e, int it) {
    const float f = t.fades[it & 3];
    stage(b ^ 1, in, it + 1);
    if (!LOCAL) keep(it);
    if constexpr (REV && !LOCAL) {
      meet(e, it);
      load_state(e, it + 2);
    }
    load(in, it + 3);
    each([&](float x, int, int) { return x * f; });
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Frag<T> fv[NT];
#pragma unroll
      for (int e = 0; e < NT; ++e) fv[e] = ld_col<VLD>(t.v(b), 32 * s, 32 * e + c0 + t.col(b));
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const Frag<T> fk = ld_col<DK>(t.key[b], 32 * s, w * (DK / 4) + 16 * m);
#pragma unroll
        for (int e = 0; e < NT; ++e) S[m] = mma(fk, fv[e], S[m]);
      }
    }
    weigh(g, it + 2);
    load_gates(g, it + 4);
    __syncthreads();
  };
  int it = 0;
  for (; it + 1 < nc; it += 2) {
    step(0, in1, g0, e0, it);
    step(1, in0, g1, e1, it + 1);
  }
  if (it < nc) step(0, in1, g0, e0, it);

  if constexpr (LOCAL) {
    float4* e = reinterpret_cast<float4*>(end_at(slot));
#pragma unroll
    for (int m = 0; m < MT; ++m) e[m] = make_float4(S[m][0], S[m][1], S[m][2], S[m][3]);
    if (split == 0 && threadIdx.x == 0) a.segG[(long)slot * a.H + h] = (float)total;
  } else {
    float* out = REV ? a.dh0 : a.ht;
    if (out && sq.piece == (REV ? 0 : segs - 1)) {
      each([&](float x, int r, int c) {
        if (r < a.dk && c < a.dv) out[sbase + (long)r * a.dv + c] = x;
        return x;
      });
    }
  }
}

// ---- outputs of a chunk ----------------------------------------------------------------
// A workgroup forms one chunk's and head's outputs from its inputs and the state that
// enters it, 64 value columns at a time.  The products are transposed: lane r16 of wave w
// has row 16 w + r16 and four consecutive columns, and the pairs' weights leave one
// product in the registers that the next one takes them from.
// Bound by what it reads, half of it the kept state where heads are 128: 4 x 4,096 tokens,
// 16 heads of 128, bf16, 403 MB in 82 us, 4.9 TB/s.  Formed inside the scan instead, every
// slice of the values forms all pairs again: 189 us for both, against 165 apart then.
template <typename T, int DK>
struct OutTiles {
  T k[DC_CH * DK], s[64 * DK], v[DC_CH * 64];
  Sums g;
};

template <typename T, int DK, bool VEC>
__global__ __launch_bounds__(256) void k_decay_out(DecayArgs a) {
  constexpr bool F32 = is_f32<T>::value;
  constexpr int KI = DK / 32;
  __shared__ __align__(16) OutTiles<T, DK> t;
  const int slot = blockIdx.x / a.H, h = blockIdx.x % a.H;
  const Slot sq = find_slot(a, slot, DC_CH);
  const int first = sq.piece * DC_CH;
  if (first >= sq.len) return;
  const int m = min(DC_CH, sq.len - first);
  const long tok = (long)sq.t0 + first;
  const int w = wave_id_s(), lane = lane_id(), r16 = lane & 15, g4 = lane >> 4, r = 16 * w + r16;
  const int dk = a.dk, dv = a.dv;
  const auto rq = head_rows<T>(a.q, tok, a.q_row, (long)(h / (a.H / a.Hq)) * dk, m, dk);
  const auto rk = head_rows<T>(a.k, tok, a.k_row, (long)(h / (a.H / a.Hk)) * dk, m, dk);
  const auto rv = head_rows<T>(a.v, tok, a.v_row, (long)(h / (a.H / a.Hv)) * dv, m, dv);
  const StateLayout<T, DK> layout(dk, dv);
  const auto rS = state_rsrc<T>(a.kept, (long)slot * a.H + h, layout.bytes);
  const auto ro = head_rows<T>(a.o, tok, (long)a.H * dv, (long)h * dv, m, dv);
  const unsigned bo = (unsigned)(a.H * dv) * (unsigned)sizeof(T);

  Gates gates;
  gates.load(a, tok, h, m);
  Piece<T, 8, VEC> pk[KI], pv[2];
  StateTile<T, DK, DK, true> ps;
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const int idx = threadIdx.x + 256 * i;
    load8(pk[i], rk, idx / (DK / 8), (unsigned)a.k_row * sizeof(T), idx % (DK / 8) * 8, dk);
  }
  Frag<T> fq[KI];
#pragma unroll
  for (int s = 0; s < KI; ++s) fq[s] = load_frag<T, VEC>(rq, 16 * w, (unsigned)a.q_row * sizeof(T), 32 * s, dk);
  auto load = [&](int v0) {  // a block of value columns
    ps.load(rS, layout, v0, 0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int idx = threadIdx.x + 256 * i;
      load8(pv[i], rv, idx / 8, (unsigned)a.v_row * sizeof(T), v0 + idx % 8 * 8, dv);
    }
  };
  auto stage = [&] {
    ps.store(t.s);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int idx = threadIdx.x + 256 * i;
      st_row8<64>(t.v, idx / 8, idx % 8 * 8, pv[i]);
    }
  };
  load(0);
  const double G = gate_sum(gates.get(a.g_head ? static_cast<const float*>(a.g)[h] : 0.f));
  if (w == 0) {
    t.g.hi[lane] = (float)G;
    t.g.lo[lane] = (float)(G - (double)(float)G);
  }
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const int idx = threadIdx.x + 256 * i;
    st_row8<DK>(t.k, idx / (DK / 8), idx % (DK / 8) * 8, pk[i]);
  }
  stage();
  __syncthreads();

  floatx4 A[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) A[i] = zero4();
#pragma unroll
  for (int s = 0; s < KI; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) A[i] = mma(ld_row<DK>(t.k, 16 * i, 32 * s), fq[s], A[i]);
  const float Gh = t.g.hi[r], Gl = t.g.lo[r];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const floatx4 f = t.g.template weights<F32>(Gh, Gl, 16 * i + 4 * g4);
#pragma unroll
    for (int e = 0; e < 4; ++e) A[i][e] = 16 * i + 4 * g4 + e <= r ? A[i][e] * f[e] : 0.f;
  }
  const Frag<T> p[2] = {frag_of<T>(A[0], A[1]), frag_of<T>(A[2], A[3])};
  const float eg = a.scale * __builtin_amdgcn_exp2f(Gh);
  for (int v0 = 0;;) {
    if (v0 + 64 < dv) load(v0 + 64);
    floatx4 oi[4], ot[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) oi[i] = ot[i] = zero4();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int s = 0; s < KI; ++s) oi[i] = mma(ld_row<DK>(t.s, 16 * i, 32 * s), fq[s], oi[i]);
#pragma unroll
      for (int s = 0; s < 2; ++s) ot[i] = mma(ld_col_acc<64>(t.v, 32 * s, 16 * i), p[s], ot[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      floatx4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(eg, oi[i][e], a.scale * ot[i][e]);
      store4c<T, VEC>(ro, r, bo, v0 + 16 * i + 4 * g4, dv, o);
    }
    v0 += 64;
    if (v0 >= dv) break;
    __syncthreads();
    stage();
    __syncthreads();
  }
}

// ---- gradients of a chunk -----------------------------------------------------------
// A workgroup forms one chunk's and head's dq, dk, dv and dg from its inputs, the state
// that enters it and the gradient of the one that leaves it.  Wave w owns the rows
// 16 w ..: of q in dq, of k and v in dk and dv.  All products are transposed, so that a
// lane holds four consecutive columns of one row.
// The chunk's four inputs lie in LDS whole; the values' tile makes room for the states',
// 64 x 64 at a time with the next one's loads in flight.
// Two workgroups a CU, eight waves, hide neither what it moves nor its LDS reads whole: 4 x
// 4,096 tokens, 16 heads of 128, bf16, 738 MB in 215 us (194 at best), 3.4 TB/s, where the
// outputs reach 4.9; a third of LDS's busy cycles are bank conflicts.
template <typename T, int DK, int DV>
struct GradTiles {
  static constexpr int VS = DV >= 128 ? DC_CH * DV : 2 * 64 * 64;
  T q[DC_CH * DK], k[DC_CH * DK], o[DC_CH * DV], vs[VS], w[DC_CH * DC_CH];
  Sums g;
  float row[DC_CH], col[4][DC_CH], far[DC_CH];
};

// A tile of 64 rows, eight columns a piece: into registers, and from there into LDS.
template <typename T, int COLS, bool VEC>
struct Rows64 {
  static constexpr int N = COLS / 32;
  Piece<T, 8, VEC> p[N];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, unsigned row_bytes, int r0, int c0, int d) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int idx = threadIdx.x + 256 * i;
      load8(p[i], rs, r0 + idx / (COLS / 8), row_bytes, c0 + idx % (COLS / 8) * 8, d);
    }
  }
  __device__ __forceinline__ void store(T* tile) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int idx = threadIdx.x + 256 * i;
      st_row8<COLS>(tile, idx / (COLS / 8), idx % (COLS / 8) * 8, p[i]);
    }
  }
};

// A row's pairs, as frag_of left them, into a tile of rows r and columns j.
template <typename T>
__device__ __forceinline__ void st_pairs(T* tile, int r, const Frag<T> (&f)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    T* d = tile + swz<64>(r, 16 * i + 4 * (lane_id() >> 4));
    if constexpr (is_f32<T>::value) {
      const float* x = f[i / 2].x + 4 * (i & 1);
      *reinterpret_cast<float4*>(d) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
      const uint4 u = __builtin_bit_cast(uint4, f[i / 2].x);
      *reinterpret_cast<uint2*>(d) = i & 1 ? make_uint2(u.z, u.w) : make_uint2(u.x, u.y);
    }
  }
}

// The pairs of a chunk, lane: row r = 16 w + r16, j = 16 i + 4 g4 + e of A (q_r . k_j) and
// B (do_r . v_j): both weighted and masked, and into col[w][t] the wave's part of the sum of
// the pairs j < t <= r for every t: over j as a product with a triangle of ones (bf16: of
// the pairs in two terms), then over the rows that remain.  Nothing is subtracted: where
// few pairs are left, row sums minus column sums would be rounding.
template <typename T, bool DG>
__device__ __forceinline__ void weigh_pairs(floatx4 (&A)[4], floatx4 (&B)[4], const Sums& g, float scale, int w, float* col) {
  constexpr bool F32 = is_f32<T>::value;
  const int lane = lane_id(), r16 = lane & 15, g4 = lane >> 4, r = 16 * w + r16;
  const float Gh = g.hi[r], Gl = g.lo[r];
  floatx4 pair[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const floatx4 wt = g.template weights<F32>(Gh, Gl, 16 * i + 4 * g4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = 16 * i + 4 * g4 + e;
      const float f = scale * wt[e], b = B[i][e] * f, x = A[i][e] * f;
      pair[i][e] = j < r ? b * A[i][e] : 0.f;
      A[i][e] = j <= r ? x : 0.f;
      B[i][e] = j <= r ? b : 0.f;
    }
  }
  if constexpr (DG) {
    floatx4 U[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) U[i] = zero4();
    floatx4 tri;
#pragma unroll
    for (int e = 0; e < 4; ++e) tri[e] = 4 * g4 + e < r16 ? 1.f : 0.f;
    const floatx4 ones = {1.f, 1.f, 1.f, 1.f};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const Frag<T> hi = frag_of<T>(pair[2 * s], pair[2 * s + 1]);
      Frag<T> lo{};
      if constexpr (!F32) {
        floatx4 x[2];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e / 4][e % 4] = pair[2 * s + e / 4][e % 4] - (float)hi.x[e];
        lo = frag_of<T>(x[0], x[1]);
      }
#pragma unroll
      for (int i = 2 * s; i < 4; ++i) {  // block i's t against blocks 2 s and 2 s + 1 of j
        const Frag<T> l = frag_of<T>(i == 2 * s ? tri : ones, i == 2 * s ? zero4() : i == 2 * s + 1 ? tri : ones);
        U[i] = mma(l, hi, U[i]);
        if constexpr (!F32) U[i] = mma(l, lo, U[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int tt = 16 * i + 4 * g4 + e;
        const float cs = sum16(r >= tt ? U[i][e] : 0.f);
        if (r16 == 0) col[tt] = cs;
      }
  }
}

template <typename T, int DK, int DV, bool VEC>
__global__ __launch_bounds__(256, sizeof(GradTiles<T, DK, DV>) <= 80 * 1024 ? 2 : 1) void k_decay_grad(DecayArgs a) {
  constexpr int KS = DK / 32, VS = DV / 32, VT = DV / 16;
  __shared__ __align__(16) GradTiles<T, DK, DV> t;
  const int slot = blockIdx.x / a.H, h = blockIdx.x % a.H;
  const Slot sq = find_slot(a, slot, DC_CH);
  const int first = sq.piece * DC_CH;
  if (first >= sq.len) return;
  const int m = min(DC_CH, sq.len - first);
  const long tok = (long)sq.t0 + first;
  const int w = wave_id_s(), lane = lane_id(), r16 = lane & 15, g4 = lane >> 4, r = 16 * w + r16;
  const int dk = a.dk, dv = a.dv;
  const StateLayout<T, DK> layout(dk, dv);
  const auto rS = state_rsrc<T>(a.kept, (long)slot * a.H + h, layout.bytes);
  const auto rD = state_rsrc<T>(a.dkept, (long)slot * a.H + h, layout.bytes);

  Gates gates;
  gates.load(a, tok, h, m);
  StateTile<T, DK, 64, true> xs;  // the states' next tiles
  StateTile<T, DK, 64, false> xd;
  {
    Rows64<T, DK, VEC> q, k;
    Rows64<T, DV, VEC> o, v;
    q.load(head_rows<T>(a.q, tok, a.q_row, (long)(h / (a.H / a.Hq)) * dk, m, dk), (unsigned)a.q_row * sizeof(T), 0, 0, dk);
    k.load(head_rows<T>(a.k, tok, a.k_row, (long)(h / (a.H / a.Hk)) * dk, m, dk), (unsigned)a.k_row * sizeof(T), 0, 0, dk);
    o.load(head_rows<T>(a.dO, tok, (long)a.H * dv, (long)h * dv, m, dv), (unsigned)(a.H * dv) * (unsigned)sizeof(T), 0, 0, dv);
    v.load(head_rows<T>(a.v, tok, a.v_row, (long)(h / (a.H / a.Hv)) * dv, m, dv), (unsigned)a.v_row * sizeof(T), 0, 0, dv);
    q.store(t.q);
    k.store(t.k);
    o.store(t.o);
    v.store(t.vs);
    xs.load(rS, layout, 0, 0);
    xd.load(rD, layout, 0, 0);
  }
  const double G = gate_sum(gates.get(a.g_head ? static_cast<const float*>(a.g)[h] : 0.f)), Gend = read_lane(G, 63);
  if (w == 0) {
    t.g.hi[lane] = (float)G;
    t.g.lo[lane] = (float)(G - (double)(float)G);
  }
  const double Gr = __shfl(G, r);
  const float eg = a.scale * __builtin_amdgcn_exp2f((float)Gr);   // of row r as a query
  const float tail = __builtin_amdgcn_exp2f((float)(Gend - Gr));  // as a key
  __syncthreads();

  // ---- the pairs
  floatx4 A[4], Bt[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) A[i] = Bt[i] = zero4();
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const Frag<T> f = ld_row<DK>(t.q, 16 * w, 32 * s);
#pragma unroll
    for (int i = 0; i < 4; ++i) A[i] = mma(ld_row<DK>(t.k, 16 * i, 32 * s), f, A[i]);
  }
  Frag<T> fv[VS];
#pragma unroll
  for (int s = 0; s < VS; ++s) {
    const Frag<T> f = ld_row<DV>(t.o, 16 * w, 32 * s);
#pragma unroll
    for (int i = 0; i < 4; ++i) Bt[i] = mma(ld_row<DV>(t.vs, 16 * i, 32 * s), f, Bt[i]);
    fv[s] = ld_row<DV>(t.vs, 16 * w, 32 * s);
  }
  if (a.dg) weigh_pairs<T, true>(A, Bt, t.g, a.scale, w, t.col[w]);
  else weigh_pairs<T, false>(A, Bt, t.g, a.scale, w, nullptr);
  const Frag<T> fp[2] = {frag_of<T>(A[0], A[1]), frag_of<T>(A[2], A[3])};
  const Frag<T> fw[2] = {frag_of<T>(Bt[0], Bt[1]), frag_of<T>(Bt[2], Bt[3])};
  st_pairs(t.w, r, fw);
  __syncthreads();
  // (the values' tile is free from here on)
  T *ts = t.vs, *td = t.vs + 64 * 64;
  xs.store(ts);
  xd.store(td);
  floatx4 iv[VT];
#pragma unroll
  for (int i = 0; i < VT; ++i) iv[i] = zero4();

  const long pq = (long)h * dk, pv = (long)h * dv;
  auto rows_of = [&](float* wide, void* out, long col, int d) {
    return wide ? head_rows<float>(wide, tok, (long)a.H * d, col, m, d) : head_rows<T>(out, tok, (long)a.H * d, col, m, d);
  };
  const auto oq = rows_of(a.pq, a.dq, pq, dk), ok = rows_of(a.pk, a.dk_, pq, dk), ov = rows_of(a.pv, a.dv_, pv, dv);
  auto put = [&](__amdgpu_buffer_rsrc_t rs, bool wide, int col, int d, const floatx4& x) {
    if (wide) store4c<float, VEC>(rs, r, (unsigned)(a.H * d) * 4u, col, d, x);
    else store4c<T, VEC>(rs, r, (unsigned)(a.H * d) * (unsigned)sizeof(T), col, d, x);
  };
  // ---- dq and dk, 64 columns at a time, and the states' part of dv
  float xr = 0.f, yj = 0.f;
#pragma unroll 1
  for (int n = 0; n < DK / 64; ++n) {
    floatx4 iq[4], ik[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) iq[i] = ik[i] = zero4();
#pragma unroll
    for (int v = 0; v < DV / 64; ++v) {
      const bool last = v + 1 == DV / 64;
      if (!last || n + 1 < DK / 64) {
        xs.load(rS, layout, last ? 0 : 64 * (v + 1), last ? 64 * (n + 1) : 64 * n);
        xd.load(rD, layout, last ? 0 : 64 * (v + 1), last ? 64 * (n + 1) : 64 * n);
      }
      __syncthreads();
      const int l = fresh_lane();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const Frag<T> fo = ld_row<DV>(t.o, 16 * w, 64 * v + 32 * s, l),
                      fk = ld_row<DK>(t.k, 16 * w, 64 * n + 32 * s, l);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          iq[i] = mma(ld_col<64>(ts, 32 * s, 16 * i, l), fo, iq[i]);
          ik[i] = mma(ld_col<64>(td, 32 * s, 16 * i, l), fv[2 * v + s], ik[i]);
          iv[4 * v + i] = mma(ld_row<64>(td, 16 * i, 32 * s, l), fk, iv[4 * v + i]);
        }
      }
      __syncthreads();
      if (!last || n + 1 < DK / 64) {
        xs.store(ts);
        xd.store(td);
      }
    }
    // the states' parts by their rows' decays, then the pairs' on top
    const int l = fresh_lane();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = 64 * n + 16 * i + 4 * (l >> 4);
      const T *qr = t.q + swz<DK>(r, col), *kr = t.k + swz<DK>(r, col);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        iq[i][e] *= eg;
        ik[i][e] *= tail;
        xr = fmaf(to_f(qr[e]), iq[i][e], xr);
        yj = fmaf(to_f(kr[e]), ik[i][e], yj);
      }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const Frag<T> f = ld_col<64>(t.w, 32 * s, 16 * w, l);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        iq[i] = mma(ld_col_acc<DK>(t.k, 32 * s, 64 * n + 16 * i, l), fw[s], iq[i]);
        ik[i] = mma(ld_col<DK>(t.q, 32 * s, 64 * n + 16 * i, l), f, ik[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      put(oq, a.pq, 64 * n + 16 * i + 4 * g4, dk, iq[i]);
      put(ok, a.pk, 64 * n + 16 * i + 4 * g4, dk, ik[i]);
    }
  }
  // ---- dv: the states' part by its rows' decays, the pairs' on top
  __syncthreads();
  st_pairs(t.w, r, fp);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < VT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) iv[i][e] *= tail;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const Frag<T> f = ld_col<64>(t.w, 32 * s, 16 * w);
#pragma unroll
    for (int i = 0; i < VT; ++i) iv[i] = mma(ld_col<DV>(t.o, 32 * s, 16 * i), f, iv[i]);
  }
#pragma unroll
  for (int i = 0; i < VT; ++i) put(ov, a.pv, 16 * i + 4 * g4, dv, iv[i]);
  // ---- dg: pairs inside the chunk, with one token before or behind it, with both
  if (!a.dg) return;
  xr = sum_groups(xr);
  yj = sum_groups(yj);
  if (g4 == 0) {
    t.row[r] = xr;
    t.far[r] = yj;
  }
  __syncthreads();
  if (w == 0) {
    const int met = 8 * decay_splits(dv);  // partial sums of the states' products
    float both = lane < met ? a.met[((long)slot * a.H + h) * met + lane] : 0.f;
    both = __builtin_amdgcn_exp2f((float)Gend) * wave_sum(both);
    const int back = 63 - lane;  // lane l holds row 63 - l: suffix sums as prefix sums
    float x = wave_prefix_sum(t.row[back]);
    float y = wave_prefix_sum(t.far[lane]);
    y = __shfl_up(y, 1);
    x = __shfl(x, back);
    const float in = ((t.col[0][lane] + t.col[1][lane]) + t.col[2][lane]) + t.col[3][lane];
    const float dg = in + x + (lane > 0 ? y : 0.f) + both;
    if (lane < m) {
      const long to = (tok + lane) * a.H + h;
      if (a.g_f32) static_cast<float*>(a.dg)[to] = dg;
      else store_elem(static_cast<bf16_t*>(a.dg) + to, dg);
    }
  }
}

// Where the inputs do not fit LDS (fp32 with heads of more than 128): the same from
// slices of 64 columns, the operands that LDS does not hold from the caches.
template <typename T>
struct WideTiles {
  T q[DC_CH * 64], k[DC_CH * 64], s[64 * 64], d[64 * 64], w[DC_CH * DC_CH], p[DC_CH * DC_CH];
  Sums g;
  float row[DC_CH], col[4][DC_CH], far[DC_CH];
};

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_decay_grad_wide(DecayArgs a) {
  __shared__ __align__(16) WideTiles<T> t;
  const int slot = blockIdx.x / a.H, h = blockIdx.x % a.H;
  const Slot sq = find_slot(a, slot, DC_CH);
  const int first = sq.piece * DC_CH;
  if (first >= sq.len) return;
  const int m = min(DC_CH, sq.len - first);
  const long tok = (long)sq.t0 + first;
  const int w = wave_id_s(), lane = lane_id(), r16 = lane & 15, g4 = lane >> 4, r = 16 * w + r16;
  const int dk = a.dk, dv = a.dv;
  const auto rq = head_rows<T>(a.q, tok, a.q_row, (long)(h / (a.H / a.Hq)) * dk, m, dk);
  const auto rk = head_rows<T>(a.k, tok, a.k_row, (long)(h / (a.H / a.Hk)) * dk, m, dk);
  const auto rv = head_rows<T>(a.v, tok, a.v_row, (long)(h / (a.H / a.Hv)) * dv, m, dv);
  const auto rdo = head_rows<T>(a.dO, tok, (long)a.H * dv, (long)h * dv, m, dv);
  const unsigned bq = (unsigned)a.q_row * sizeof(T), bk = (unsigned)a.k_row * sizeof(T),
                 bv = (unsigned)a.v_row * sizeof(T), bo = (unsigned)(a.H * dv) * (unsigned)sizeof(T);
  typedef StateLayout<T, 256> Layout;  // (fp32: the same for every size)
  const Layout layout(dk, dv);
  const auto rS = state_rsrc<T>(a.kept, (long)slot * a.H + h, layout.bytes);
  const auto rD = state_rsrc<T>(a.dkept, (long)slot * a.H + h, layout.bytes);

  Gates gates;
  gates.load(a, tok, h, m);
  const double G = gate_sum(gates.get(a.g_head ? static_cast<const float*>(a.g)[h] : 0.f)), Gend = read_lane(G, 63);
  if (w == 0) {
    t.g.hi[lane] = (float)G;
    t.g.lo[lane] = (float)(G - (double)(float)G);
  }
  const float eg = a.scale * __builtin_amdgcn_exp2f((float)__shfl(G, r));        // of row r as a query
  const float tail = __builtin_amdgcn_exp2f((float)(Gend - __shfl(G, r)));       // as a key
  __syncthreads();

  // ---- the pairs' products (q_r . k_j) and (do_r . v_j), lane: row r, j = 16 i + 4 g4 + e
  floatx4 A[4], Bt[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) A[i] = Bt[i] = zero4();
  for (int s = 0; s < dk; s += 32) {
    const Frag<T> f = load_frag<T, VEC>(rq, 16 * w, bq, s, dk);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i <= w) A[i] = mma(load_frag<T, VEC>(rk, 16 * i, bk, s, dk), f, A[i]);
  }
  for (int s = 0; s < dv; s += 32) {
    const Frag<T> f = load_frag<T, VEC>(rdo, 16 * w, bo, s, dv);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i <= w) Bt[i] = mma(load_frag<T, VEC>(rv, 16 * i, bv, s, dv), f, Bt[i]);
  }
  if (a.dg) weigh_pairs<T, true>(A, Bt, t.g, a.scale, w, t.col[w]);
  else weigh_pairs<T, false>(A, Bt, t.g, a.scale, w, nullptr);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    st_row4<64>(t.p, r, 16 * i + 4 * g4, A[i]);
    st_row4<64>(t.w, r, 16 * i + 4 * g4, Bt[i]);
  }
  const Frag<T> fw[2] = {frag_of<T>(Bt[0], Bt[1]), frag_of<T>(Bt[2], Bt[3])};

  // ---- dq and dk, 64 columns at a time
  float xr = 0.f, yj = 0.f;
  const long pq = (long)h * dk, pv = (long)h * dv;
  const auto oq = a.pq ? head_rows<float>(a.pq, tok, (long)a.H * dk, pq, m, dk)
                       : head_rows<T>(a.dq, tok, (long)a.H * dk, pq, m, dk);
  const auto ok = a.pk ? head_rows<float>(a.pk, tok, (long)a.H * dk, pq, m, dk)
                       : head_rows<T>(a.dk_, tok, (long)a.H * dk, pq, m, dk);
  const auto ov = a.pv ? head_rows<float>(a.pv, tok, (long)a.H * dv, pv, m, dv)
                       : head_rows<T>(a.dv_, tok, (long)a.H * dv, pv, m, dv);
  auto put = [&](__amdgpu_buffer_rsrc_t rs, bool wide, int col, int d, const floatx4& x) {
    if (wide) store4c<float, VEC>(rs, r, (unsigned)(a.H * d) * 4u, col, d, x);
    else store4c<T, VEC>(rs, r, (unsigned)(a.H * d) * (unsigned)sizeof(T), col, d, x);
  };
  for (int c0 = 0; c0 < dk; c0 += 64) {
    Piece<T, 8, VEC> x[2], y[2];
    StateTile<T, 256, 64, true> xs;
    StateTile<T, 256, 64, false> xd;
    auto tile = [&](__amdgpu_buffer_rsrc_t rs, unsigned rb, int r0, int c, int d, Piece<T, 8, VEC>(&p)[2]) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int idx = threadIdx.x + 256 * i;
        load8(p[i], rs, r0 + idx / 8, rb, c + idx % 8 * 8, d);
      }
    };
    auto put_tile = [&](T* to, const Piece<T, 8, VEC>(&p)[2]) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int idx = threadIdx.x + 256 * i;
        st_row8<64>(to, idx / 8, idx % 8 * 8, p[i]);
      }
    };
    tile(rq, bq, 0, c0, dk, x);
    tile(rk, bk, 0, c0, dk, y);
    __syncthreads();
    put_tile(t.q, x);
    put_tile(t.k, y);
    floatx4 aq[4], ak[4], iq[4], ik[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) aq[i] = ak[i] = iq[i] = ik[i] = zero4();
    for (int v0 = 0; v0 < dv; v0 += 64) {
      xs.load(rS, layout, v0, c0);
      xd.load(rD, layout, v0, c0);
      Frag<T> fo[2], fv[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        fo[s] = load_frag<T, VEC>(rdo, 16 * w, bo, v0 + 32 * s, dv);
        fv[s] = load_frag<T, VEC>(rv, 16 * w, bv, v0 + 32 * s, dv);
      }
      if (v0 > 0) __syncthreads();
      xs.store(t.s);
      xd.store(t.d);
      __syncthreads();
      if (v0 == 0) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const Frag<T> f = ld_col<64>(t.w, 32 * s, 16 * w);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            aq[i] = mma(ld_col_acc<64>(t.k, 32 * s, 16 * i), fw[s], aq[i]);
            ak[i] = mma(ld_col<64>(t.q, 32 * s, 16 * i), f, ak[i]);
          }
        }
      }
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          iq[i] = mma(ld_col<64>(t.s, 32 * s, 16 * i), fo[s], iq[i]);
          ik[i] = mma(ld_col<64>(t.d, 32 * s, 16 * i), fv[s], ik[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = 16 * i + 4 * g4;
      const T *qr = t.q + swz<64>(r, col), *kr = t.k + swz<64>(r, col);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x1 = eg * iq[i][e], y1 = tail * ik[i][e];
        xr = fmaf(to_f(qr[e]), x1, xr);
        yj = fmaf(to_f(kr[e]), y1, yj);
        aq[i][e] += x1;
        ak[i][e] += y1;
      }
      put(oq, a.pq, c0 + col, dk, aq[i]);
      put(ok, a.pk, c0 + col, dk, ak[i]);
    }
  }
  // ---- dv, 64 columns at a time
  // rows v .. of the state's gradient, eight columns from s + 8 g4: two of a lane's pieces
  auto state_frag = [&](int v, int s) {
    const int col = s + 8 * g4;
    Frag<T> f;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const auto u = __builtin_amdgcn_raw_buffer_load_b128(
          rD, layout.at(v / 16, col / 16, (col % 16 / 4 + half) * 16 + r16), 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) f.x[4 * half + e] = __uint_as_float(u[e]);
    }
    return f;
  };
  for (int v0 = 0; v0 < dv; v0 += 64) {
    Piece<T, 8, VEC> x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int idx = threadIdx.x + 256 * i;
      load8(x[i], rdo, idx / 8, bo, v0 + idx % 8 * 8, dv);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int idx = threadIdx.x + 256 * i;
      st_row8<64>(t.q, idx / 8, idx % 8 * 8, x[i]);
    }
    floatx4 av[4], iv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) av[i] = iv[i] = zero4();
    for (int s = 0; s < dk; s += 32) {
      const Frag<T> f = load_frag<T, VEC>(rk, 16 * w, bk, s, dk);
#pragma unroll
      for (int i = 0; i < 4; ++i) iv[i] = mma(state_frag(v0 + 16 * i, s), f, iv[i]);
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const Frag<T> f = ld_col<64>(t.p, 32 * s, 16 * w);
#pragma unroll
      for (int i = 0; i < 4; ++i) av[i] = mma(ld_col<64>(t.q, 32 * s, 16 * i), f, av[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      floatx4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(tail, iv[i][e], av[i][e]);
      put(ov, a.pv, v0 + 16 * i + 4 * g4, dv, o);
    }
  }
  // ---- dg: pairs inside the chunk, with one token before or behind it, with both
  if (!a.dg) return;
  xr = sum_groups(xr);
  yj = sum_groups(yj);
  if (g4 == 0) {
    t.row[r] = xr;
    t.far[r] = yj;
  }
  __syncthreads();
  if (w == 0) {
    const int met = 8 * decay_splits(dv);  // partial sums of the states' products
    float both = lane < met ? a.met[((long)slot * a.H + h) * met + lane] : 0.f;
    both = __builtin_amdgcn_exp2f((float)Gend) * wave_sum(both);
    const int back = 63 - lane;  // lane l holds row 63 - l: suffix sums as prefix sums
    float x = wave_prefix_sum(t.row[back]);
    float y = wave_prefix_sum(t.far[lane]);
    y = __shfl_up(y, 1);
    x = __shfl(x, back);
    const float in = ((t.col[0][lane] + t.col[1][lane]) + t.col[2][lane]) + t.col[3][lane];
    const float dg = in + x + (lane > 0 ? y : 0.f) + both;
    if (lane < m) {
      const long to = (tok + lane) * a.H + h;
      if (a.g_f32) static_cast<float*>(a.dg)[to] = dg;
      else store_elem(static_cast<bf16_t*>(a.dg) + to, dg);
    }
  }
}

// Gradients of shared heads: the sum over the state heads that share one, in their order.
// Four values a thread where the head's size allows (bf16, 16,384 tokens, 16 heads of 64 in
// fp32 to 4: 14 us, 5.4 TB/s with what the caches hold; value by value 22).
template <typename T, int C>
__global__ __launch_bounds__(256) void k_decay_shared(const float* __restrict__ p, T* __restrict__ out,
                                                      const int32_t* __restrict__ cu, int S, int Ttot, int heads, int per,
                                                      int d) {
  // (rows outside the sequences have no gradients and are left as they are)
  const long row = (long)heads * d / C;
  const long from_row = cu ? min(max(cu[0], 0), Ttot) : 0, to_row = cu ? min(max(cu[S], 0), Ttot) : Ttot;
  const long n = to_row * row;
  for (long i = from_row * row + (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
    const unsigned w = (unsigned)(d / C);
    const long head = i / w;
    const float* from = p + head * per * d + (i - head * w) * C;
    float s[C];
#pragma unroll
    for (int e = 0; e < C; ++e) s[e] = 0.f;
#pragma unroll 4
    for (int k = 0; k < per; ++k) {
      Piece<float, C, true> x;
      x.load(from + (long)k * d, C);
#pragma unroll
      for (int e = 0; e < C; ++e) s[e] += x.get(e);
    }
    store_piece<T, C, true>(out + i * C, s, C);
  }
}

// ---- one token -----------------------------------------------------------------------
// Bound by the state, read and written once.  A workgroup takes COLS groups of C value
// columns of one row and head; thread (i, c) the key rows i, i + 256 / COLS, ...
// 200 rows, 16 heads of 128: 423 MB in 83 us, 5.1 TB/s (a part stays in the on-die cache).
template <typename T, int C, int COLS>
__global__ __launch_bounds__(256) void k_decay_step(DecayArgs a) {
  constexpr int RG = 256 / COLS;
  __shared__ float ks[256], qs[256], red[RG][COLS * C];
  const int b = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, c = tid % COLS, rg = tid / COLS;
  const int col = (blockIdx.z * COLS + c) * C;
  const long slot = a.slots ? a.slots[b] : b;
  T* o = static_cast<T*>(a.o) + ((long)b * a.H + h) * a.dv;
  if (slot < 0 || slot >= a.num_slots) {  // padding
    if (rg == 0)
      for (int i = 0; i < C; ++i)
        if (col + i < a.dv) store_elem(o + col + i, 0.f);
    return;
  }
  const T* k = static_cast<const T*>(a.k) + b * a.k_row + (long)(h / (a.H / a.Hk)) * a.dk;
  const T* q = static_cast<const T*>(a.q) + b * a.q_row + (long)(h / (a.H / a.Hq)) * a.dk;
  const T* v = static_cast<const T*>(a.v) + b * a.v_row + (long)(h / (a.H / a.Hv)) * a.dv;
  float g = gate_of(a, b, h);
  g = g < -128.f ? -128.f : g;
  const float alpha = __builtin_amdgcn_exp2f(LOG2E * g);
  ks[tid] = tid < a.dk ? to_f(k[tid]) : 0.f;
  qs[tid] = tid < a.dk ? to_f(q[tid]) : 0.f;
  float vv[C], acc[C];
#pragma unroll
  for (int i = 0; i < C; ++i) {
    vv[i] = col + i < a.dv ? to_f(v[col + i]) : 0.f;
    acc[i] = 0.f;
  }
  __syncthreads();
  float* S = a.state + (slot * a.H + h) * (long)a.dk * a.dv + col;
  if (col < a.dv) {
#pragma unroll 8
    for (int r = rg; r < a.dk; r += RG) {
      float* p = S + (long)r * a.dv;
      float x[C];
      if constexpr (C == 4) {
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        const f32x4 s = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
        f32x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = x[i] = fmaf(alpha, s[i], ks[r] * vv[i]);
        __builtin_nontemporal_store(y, reinterpret_cast<f32x4*>(p));
      } else {
        x[0] = fmaf(alpha, *p, ks[r] * vv[0]);
        *p = x[0];
      }
#pragma unroll
      for (int i = 0; i < C; ++i) acc[i] = fmaf(qs[r], x[i], acc[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < C; ++i) red[rg][c * C + i] = acc[i];
  __syncthreads();
  const int out = blockIdx.z * COLS * C + tid;
  if (tid < COLS * C && out < a.dv) {
    float s = 0.f;
    for (int i = 0; i < RG; ++i) s += red[i][tid];
    store_elem(o + out, a.scale * s);
  }
}

// ---- launches --------------------------------------------------------------------------
template <typename T>
static bool pieces8(const void* p, long row, int d) {
  return d % 8 == 0 && (uintptr_t)p % 16 == 0 && row % (16 / (long)sizeof(T)) == 0;
}

template <typename T, bool REV, bool LOCAL, bool VEC>
static hipError_t run_scan(const DecayArgs& a) {
  const long units = decay_slots(a, a.seglen) * a.H, ns = decay_splits(a.dv);
  if (units == 0) return hipSuccess;
  const long grid = (units + 7) / 8 * 8 * ns;
  if (grid > INT32_MAX / SCAN_THREADS) return hipErrorInvalidValue;
  switch (decay_dkp(a.dk)) {
    case 64: k_decay_scan<T, 64, REV, LOCAL, VEC><<<(unsigned)grid, SCAN_THREADS, 0, a.stream>>>(a, (int)units); break;
    case 128: k_decay_scan<T, 128, REV, LOCAL, VEC><<<(unsigned)grid, SCAN_THREADS, 0, a.stream>>>(a, (int)units); break;
    default: k_decay_scan<T, 256, REV, LOCAL, VEC><<<(unsigned)grid, SCAN_THREADS, 0, a.stream>>>(a, (int)units); break;
  }
  return hipGetLastError();
}
template <typename T, bool REV, bool VEC>
static hipError_t run_scans(const DecayArgs& a) {
  if (a.segS) {
    const hipError_t e = run_scan<T, REV, true, VEC>(a);
    if (e != hipSuccess) return e;
  }
  return run_scan<T, REV, false, VEC>(a);
}

template <typename T, bool VEC>
static hipError_t run_out(const DecayArgs& a) {
  if (a.Ttot == 0) return hipSuccess;
  const unsigned grid = (unsigned)(decay_slots(a, DC_CH) * a.H);
  switch (decay_dkp(a.dk)) {
    case 64: k_decay_out<T, 64, VEC><<<grid, 256, 0, a.stream>>>(a); break;
    case 128: k_decay_out<T, 128, VEC><<<grid, 256, 0, a.stream>>>(a); break;
    default: k_decay_out<T, 256, VEC><<<grid, 256, 0, a.stream>>>(a); break;
  }
  return hipGetLastError();
}
template <typename T>
static hipError_t run_fwd(const DecayArgs& a) {
  const bool vec = pieces8<T>(a.q, a.q_row, a.dk) && pieces8<T>(a.k, a.k_row, a.dk) && pieces8<T>(a.v, a.v_row, a.dv) &&
                   pieces8<T>(a.o, (long)a.H * a.dv, a.dv);
  const hipError_t e = vec ? run_scans<T, false, true>(a) : run_scans<T, false, false>(a);
  if (e != hipSuccess) return e;
  return vec ? run_out<T, true>(a) : run_out<T, false>(a);
}
hipError_t launch_decay_fwd(const DecayArgs& a) { return a.bf16 ? run_fwd<bf16_t>(a) : run_fwd<float>(a); }

template <typename T>
static hipError_t run_shared(const DecayArgs& a, const float* p, void* out, int heads, int d) {
  const int c = d % 4 == 0 && (uintptr_t)out % (4 * sizeof(T)) == 0 ? 4 : 1;
  const long blocks = ((long)a.Ttot * heads * d / c + 255) / 256;
  const unsigned grid = (unsigned)(blocks < 16384 ? blocks : 16384);
  if (c == 4) k_decay_shared<T, 4><<<grid, 256, 0, a.stream>>>(p, static_cast<T*>(out), a.cu_seqlens, a.S, a.Ttot, heads, a.H / heads, d);
  else k_decay_shared<T, 1><<<grid, 256, 0, a.stream>>>(p, static_cast<T*>(out), a.cu_seqlens, a.S, a.Ttot, heads, a.H / heads, d);
  return hipGetLastError();
}
template <typename T, int DK, bool VEC>
static void grad_of(const DecayArgs& a, unsigned grid) {
  switch (decay_dkp(a.dv)) {
    case 64: k_decay_grad<T, DK, 64, VEC><<<grid, 256, 0, a.stream>>>(a); break;
    case 128: k_decay_grad<T, DK, 128, VEC><<<grid, 256, 0, a.stream>>>(a); break;
    default:
      if constexpr (!is_f32<T>::value) k_decay_grad<T, DK, 256, VEC><<<grid, 256, 0, a.stream>>>(a);
  }
}
template <typename T, bool VEC>
static hipError_t run_grad(const DecayArgs& a, unsigned grid) {
  if constexpr (is_f32<T>::value) {
    if (a.dk > 128 || a.dv > 128) {
      k_decay_grad_wide<T, VEC><<<grid, 256, 0, a.stream>>>(a);
      return hipGetLastError();
    }
  }
  switch (decay_dkp(a.dk)) {
    case 64: grad_of<T, 64, VEC>(a, grid); break;
    case 128: grad_of<T, 128, VEC>(a, grid); break;
    default:
      if constexpr (!is_f32<T>::value) grad_of<T, 256, VEC>(a, grid);
  }
  return hipGetLastError();
}
template <typename T>
static hipError_t run_bwd(const DecayArgs& a) {
  const bool vec = pieces8<T>(a.q, a.q_row, a.dk) && pieces8<T>(a.k, a.k_row, a.dk) && pieces8<T>(a.v, a.v_row, a.dv) &&
                   pieces8<T>(a.dO, (long)a.H * a.dv, a.dv) && pieces8<T>(a.dq, 0, a.dk) &&
                   pieces8<T>(a.dk_, 0, a.dk) && pieces8<T>(a.dv_, 0, a.dv);
  hipError_t e = vec ? run_scans<T, true, true>(a) : run_scans<T, true, false>(a);
  if (e != hipSuccess || a.Ttot == 0) return e;
  const long grid = decay_slots(a, DC_CH) * a.H;
  if (grid > INT32_MAX / 256) return hipErrorInvalidValue;
  e = vec ? run_grad<T, true>(a, (unsigned)grid) : run_grad<T, false>(a, (unsigned)grid);
  if (e == hipSuccess && a.pq) e = run_shared<T>(a, a.pq, a.dq, a.Hq, a.dk);
  if (e == hipSuccess && a.pk) e = run_shared<T>(a, a.pk, a.dk_, a.Hk, a.dk);
  if (e == hipSuccess && a.pv) e = run_shared<T>(a, a.pv, a.dv_, a.Hv, a.dv);
  return e;
}
hipError_t launch_decay_bwd(const DecayArgs& a) { return a.bf16 ? run_bwd<bf16_t>(a) : run_bwd<float>(a); }

template <typename T>
static hipError_t run_step(const DecayArgs& a) {
  if (a.S == 0) return hipSuccess;
  const bool vec = a.dv % 4 == 0 && (uintptr_t)a.state % 16 == 0;
  auto grid = [&](int cols) { return dim3(a.S, a.H, (a.dv + cols - 1) / cols); };
  // few states: slices of 32 columns give more workgroups, so more CUs stream the states
  if (!vec) k_decay_step<T, 1, 32><<<grid(32), 256, 0, a.stream>>>(a);
  else if ((long)a.S * a.H * ((a.dv + 127) / 128) < 1024) k_decay_step<T, 4, 8><<<grid(32), 256, 0, a.stream>>>(a);
  else k_decay_step<T, 4, 32><<<grid(128), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}
hipError_t launch_decay_step(const DecayArgs& a) { return a.bf16 ? run_step<bf16_t>(a) : run_step<float>(a); }

}  // namespace comba
