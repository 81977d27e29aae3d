// Selective state space scan: per channel c and state n
//
//   h_t = exp(dt_t A) h_{t-1} + dt_t u_t B_t,   s_t = <C_t, h_t> + Dskip u_t,   y_t = s_t silu(z_t)
//
// A decay of its own for every (channel, state, token) leaves nothing for the
// matrix units: the work is one exponential (two issue slots) and four vector
// operations per (channel, state, token), and these, not the bytes, bound every
// long call.  4 x 4,096 tokens, 4,096 channels, 16 states, gated, bf16: forward 352
// us with 10 vector instructions per (channel, state, token), the vector units busy
// 88% of the time (its bytes alone would take 108 us); backward 936 us, with 25 and
// 84% in its main kernel and 50 us of it for the sums.
//
// Layout of a wave: CW channels x N states.  A lane holds CPL = 2 channels x 4
// states (lane group ng = lane / CG takes states 4 ng .. 4 ng + 3, lane cg = lane
// % CG takes channels CPL cg ..), so that sums over states are three in-lane
// adds and log2(N / 4) lane exchanges for CPL channels at once, and sums over
// channels (the gradients of B and C) start with in-lane adds as well.
//
// Time: a workgroup's W waves take consecutive chunks of L tokens of a tile.  A
// wave forms its chunk's decays once and keeps them in registers, with the
// chunk's state and outputs from a zero start; the chunks' (product of decays,
// state) pairs are combined through LDS, each state by the thread that owns it,
// and a second pass adds what the true state gives, with the kept decays.  The
// second pass costs two operations more per value than a walk token by token,
// but leaves W times as many waves.  Twelve waves are three a SIMD at 168
// registers: forward 356 us, with eight 408, with six and two workgroups a CU 549.
//
// Eleven of the variants need more than 168 and keep 3 to 10 registers in scratch: the
// gated fp32 backward of 16 states, the backward of 32 states (but ungated, aligned
// bf16), the gated backward and the gated fp32 forward of 16 states for unaligned
// rows.  Their scratch stays in the caches (the fp32 backward of 16 states writes 1,033
// MiB, its results and partial sums 1,024), and they issue as densely (80 to 83% busy).
// 4 x 4,096 tokens, 4,096 channels, gated, us of the calls, forward and backward: 8 states
// bf16 235 and 594, fp32 267 and 613; 16 states 363 and 954, fp32 377 and 970; 32 states
// 669 and 2,072, fp32 681 and 2,141; rows off by one element: 16 states 462 and 1,033, fp32
// 494 and 1,157; 32 states 862 and 2,294, fp32 780 and 2,235; 8 states 346 and 771.
#include "comba_layer_device.hpp"
#include "comba_layer_launch.h"

namespace comba {

// Channels of a lane: four would double the kept decays, and spill.
constexpr int SEL_CPL = 2;
// Waves of a forward workgroup: three a SIMD, where the registers suffice.
constexpr int sel_waves(int N) { return N == 8 ? 8 : 12; }

template <int N, int CPL>
struct SelTile {
  static constexpr int LN = N / 4;     // lane groups over the states
  static constexpr int CG = 64 / LN;   // lanes over the channels
  static constexpr int CW = CG * CPL;  // channels of a wave
  static constexpr int NE = CW * N;    // states of a wave, 4 CPL per lane
  static constexpr int LOW = LN == 2 ? 5 : LN == 4 ? 4 : 3;  // lowest lane bit of the state group
  static_assert(LN == 2 || LN == 4 || LN == 8, "states per channel");
};

// C consecutive floats of LDS.
template <int C>
__device__ __forceinline__ void lds_get(const float* p, float (&v)[C]) {
  if constexpr (C == 4) {
    const float4 f = *reinterpret_cast<const float4*>(p);
    v[0] = f.x;
    v[1] = f.y;
    v[2] = f.z;
    v[3] = f.w;
  } else if constexpr (C == 2) {
    const float2 f = *reinterpret_cast<const float2*>(p);
    v[0] = f.x;
    v[1] = f.y;
  } else {
    v[0] = p[0];
  }
}
template <int C>
__device__ __forceinline__ void lds_put(float* p, const float (&v)[C]) {
  if constexpr (C == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else if constexpr (C == 2) {
    *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
  } else {
    p[0] = v[0];
  }
}

// p[c], or 0 without p: loaded without a branch (which would be waited for on the
// spot) from `any`, which has as many values.
__device__ __forceinline__ float or_zero(const float* p, const float* any, int c) {
  const float v = (p ? p : any)[c];
  return p ? v : 0.f;
}

// What a workgroup works on: a work row (a segment of a sequence) and a block of CW
// channels of one group.  Two neighbouring blocks, which share the 128-byte lines
// of their rows, go to workgroups eight apart and so to the same XCD.
struct SelBlock {
  int seq, seg, blk, g;  // sequence, its segment, channel block (of all groups), group
  int row0;              // the work row of the sequence's first segment
  int c0, cend;          // channels [c0, cend)
  int tok0, len;         // the sequence's tokens
  int t0, t1;            // the segment's tokens, counted in the sequence
  int nseg;              // the sequence's segments (at least one)
};
template <int CW>
__device__ __forceinline__ SelBlock sel_block(const SelectArgs& a, const SelectRows& q) {
  const int Dg = a.D / a.G, nblk = (Dg + CW - 1) / CW, nb = a.G * nblk;
  int b = blockIdx.x;
  if ((b | 15) < (int)gridDim.x) b = (b & ~15) | ((b & 7) << 1) | ((b >> 3) & 1);
  SelBlock s;
  const int r = b / nb, l = lane_id();
  int most = 1;  // segments that have a work row
  s.blk = b - r * nb;
  if (q.n > 0) {
    const int at = l < q.n ? q.at[l] : INT32_MAX, seq = l < q.n ? q.seq[l] : INT32_MAX;
    const int listed = q.at[q.n];
    if (r < listed) {
      const int i = __builtin_popcountll(__ballot(at <= r)) - 1;
      s.row0 = __builtin_amdgcn_readlane(at, i);
      s.seq = __builtin_amdgcn_readlane(seq, i);
      most = (i + 1 < q.n ? __builtin_amdgcn_readlane(at, i + 1) : listed) - s.row0;
    } else {  // the (r - listed)-th of the others
      s.row0 = r;
      s.seq = r - listed;
      for (int k = 0; k < SEL_LIST; ++k) s.seq = r - listed + __builtin_popcountll(__ballot(seq <= s.seq));
    }
  } else {
    s.seq = r / a.segs;
    s.row0 = s.seq * a.segs;
    most = a.segs;
    if (a.cu_seqlens && a.S > 1 && a.S <= 64) {
      // no host offsets: lane l ranks sequence l by its length
      const int n = l < a.S ? a.cu_seqlens[l + 1] - a.cu_seqlens[l] : 0;
      int rank = 0;
      for (int j = 0; j < a.S; ++j) {
        const int m = __builtin_amdgcn_readlane(n, j);
        rank += m > n || (m == n && j < l);
      }
      s.seq = __builtin_ctzll(__ballot(l < a.S && rank == r));
    }
  }
  s.seg = r - s.row0;
  s.g = s.blk / nblk;
  s.c0 = s.g * Dg + (s.blk - s.g * nblk) * CW;
  s.cend = min(s.c0 + CW, (s.g + 1) * Dg);
  int t1;
  seq_range(a.cu_seqlens, s.seq, a.Tseq, a.Ttot, s.tok0, t1);
  s.len = t1 - s.tok0;
  const bool cut = most > 1 && s.len > a.segmin;
  s.nseg = cut ? min((s.len + a.seglen - 1) / a.seglen, most) : 1;
  s.t0 = cut ? min(s.len, s.seg * a.seglen) : (s.seg > 0 ? s.len : 0);
  s.t1 = cut ? min(s.len, s.t0 + a.seglen) : s.len;
  return s;
}

// The state that thread `slot` of the exchange owns, as (channel in the block,
// state): slot = (i * 64 + lane) * 4 + j is the lane's channel i, state j.
template <int N, int CPL>
__device__ __forceinline__ void sel_slot(int slot, int& ch, int& n) {
  using S = SelTile<N, CPL>;
  const int i = slot / 256, l = (slot >> 2) & 63, j = slot & 3;
  ch = (l % S::CG) * CPL + i;
  n = (l / S::CG) * 4 + j;
}

// A segment's end from a zero start, for rows cut into segments: its final state
// (REV: the decayed gradient of the state that enters it) and, per channel, the
// sum of its steps, whose exponential is the segment's decay product.  Without
// outputs and second pass: half the forward's time per token (12,600 tokens of
// 2,048 channels, 16 states: 99 us), a quarter of the backward's.
template <typename Tin, int N, int CPL, bool VEC, bool REV>
__global__ __launch_bounds__(64 * sel_waves(N)) void k_select_seg(SelectArgs a, SelectRows q) {
  constexpr int L = 8, W = sel_waves(N);
  using S = SelTile<N, CPL>;
  constexpr int LN = S::LN, CG = S::CG, CW = S::CW, NE = S::NE, TL = L / LN, TILE = L * W;
  constexpr int NB = L * N / 64;
  constexpr unsigned EB = sizeof(Tin);
  static_assert(L % LN == 0 && N % NB == 0, "tile");
  struct WaveLds {
    float dt[L][CW], x[L][CW], R[L][N];  // x R: dt u B, or gy C
  };
  __shared__ __align__(16) WaveLds lds[W];
  __shared__ __align__(16) float ex[W][2][NE];

  const SelBlock sb = sel_block<CW>(a, q);
  // the last segment's end is nobody's start (REV: the first one's)
  if (sb.t0 >= sb.t1 || sb.seg == (REV ? 0 : sb.nseg - 1)) return;
  const int lane = lane_id(), w = wave_id_s(), ng = lane / CG, cg = lane % CG;
  const int cl = sb.c0 + cg * CPL, nv = max(0, min(CPL, sb.cend - cl));
  WaveLds& my = lds[w];
  const bool gate = REV && a.z;

  const unsigned tok = w * L + ng, cb = nv > 0 ? (unsigned)cl * EB : BUF_OOB;
  const long xrow = REV ? a.D : a.u_row, rrow = REV ? a.c_row : a.b_row;
  const unsigned xb = xrow * EB, db = a.delta_row * EB, zb = a.z_row * EB;
  const unsigned xo = tok * xb + cb, dof = tok * db + cb, zo = tok * zb + cb;
  const int bt = lane * NB / N, bs = lane * NB % N;
  const unsigned ro = (w * L + bt) * (unsigned)(rrow * EB) + (sb.g * N + bs) * EB;
  const int tiles = (sb.t1 - sb.t0 + TILE - 1) / TILE, dir = REV ? -TILE : TILE;
  const long row0 = sb.tok0 + sb.t0 + (REV ? (long)(tiles - 1) * TILE : 0);
  RowsAt tx(REV ? a.dy : a.u, row0, xb), td(a.delta, row0, db), tz(a.z, row0, zb);
  RowsAt tr(REV ? a.Cm : a.Bm, row0, rrow * EB);
  Piece<Tin, CPL, VEC> px[TL], pd[TL], pz[TL];
  Piece<Tin, NB, VEC> pr;
  auto load = [&](int tile) {  // in the order of the walk
    const int rows = min(sb.t1 - sb.t0 - (REV ? tiles - 1 - tile : tile) * TILE, TILE);
    const auto rx = tx.rows(rows), rd = td.rows(rows), rr = tr.rows(rows);
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      px[k].load(rx, xo + k * LN * xb, nv);
      pd[k].load(rd, dof + k * LN * db, nv);
    }
    if (gate) {
      const auto rz = tz.rows(rows);
#pragma unroll
      for (int k = 0; k < TL; ++k) pz[k].load(rz, zo + k * LN * zb, nv);
    }
    pr.load(rr, ro, NB);
    tx.step(dir);
    td.step(dir);
    if (gate) tz.step(dir);
    tr.step(dir);
  };
  load(0);

  float A2[CPL][4], bias[CPL], total[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = i < nv ? cl + i : sb.c0;
    bias[i] = or_zero(a.bias, a.A, c);
    total[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v = a.A[(long)c * N + ng * 4 + j];
      A2[i][j] = i < nv ? v * LOG2E : 0.f;
    }
  }
  const int own = threadIdx.x;  // the state that this thread owns, below NE
  float H = 0.f;
  for (int tile = 0; tile < tiles; ++tile) {
    const int t0 = sb.t0 + (REV ? tiles - 1 - tile : tile) * TILE + w * L;
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      const int tl = ng + LN * k;
      const bool ok = t0 + tl < sb.t1;
      float dt[CPL], x[CPL];
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        dt[i] = pd[k].get(i) + bias[i];
        x[i] = px[k].get(i);
      }
      if (a.softplus) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) dt[i] = softplus_acc(dt[i]);
      }
      if (gate) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
          const float zv = pz[k].get(i);
          x[i] *= zv * sigmoid_acc(zv);
        }
      }
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        dt[i] = ok ? dt[i] : 0.f;
        if constexpr (!REV) x[i] *= dt[i];
        total[i] += dt[i];
      }
      lds_put<CPL>(&my.dt[tl][cg * CPL], dt);
      lds_put<CPL>(&my.x[tl][cg * CPL], x);
    }
    {
      float v[NB];
#pragma unroll
      for (int e = 0; e < NB; ++e) v[e] = pr.get(e);
      lds_put<NB>(&my.R[bt][bs], v);
    }
    __builtin_amdgcn_wave_barrier();
    if (tile + 1 < tiles) load(tile + 1);
    float h[CPL][4], sdt[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      sdt[i] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) h[i][j] = 0.f;
    }
#pragma unroll
    for (int tt = 0; tt < L; ++tt) {
      const int t = REV ? L - 1 - tt : tt;
      float dt[CPL], x[CPL], Rv[4];
      lds_get<CPL>(&my.dt[t][cg * CPL], dt);
      lds_get<CPL>(&my.x[t][cg * CPL], x);
      lds_get<4>(&my.R[t][ng * 4], Rv);
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        sdt[i] += dt[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float d = __builtin_amdgcn_exp2f(dt[i] * A2[i][j]);
          if constexpr (REV) h[i][j] = d * fmaf(x[i], Rv[j], h[i][j]);
          else h[i][j] = fmaf(d, h[i][j], x[i] * Rv[j]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      float p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = __builtin_amdgcn_exp2f(sdt[i] * A2[i][j]);
      lds_put<4>(&ex[w][0][(i * 64 + lane) * 4], p);
      lds_put<4>(&ex[w][1][(i * 64 + lane) * 4], h[i]);
    }
    __syncthreads();
    if (own < NE) {
#pragma unroll
      for (int mm = 0; mm < W; ++mm) {
        const int m = REV ? W - 1 - mm : mm;
        H = fmaf(ex[m][0][own], H, ex[m][1][own]);
      }
    }
    __syncthreads();
  }
  const long at = (long)(sb.row0 + sb.seg) * a.D;
  int oc, on;
  sel_slot<N, CPL>(own, oc, on);
  if (own < NE && sb.c0 + oc < sb.cend) a.segF[(at + sb.c0 + oc) * N + on] = H;
  // the steps' sum: over the lane groups and waves, which held different tokens
  float* red = &ex[0][0][0];
#pragma unroll
  for (int i = 0; i < CPL; ++i) red[(w * CPL + i) * 64 + lane] = total[i];
  __syncthreads();
  const int ch = threadIdx.x;
  if (ch < CW && sb.c0 + ch < sb.cend) {
    float v = 0.f;
    for (int m = 0; m < W; ++m)
      for (int e = 0; e < LN; ++e) v += red[(m * CPL + ch % CPL) * 64 + e * CG + ch / CPL];
    a.segdt[at + sb.c0 + ch] = v;
  }
}

// The state (REV: its gradient) that enters a segment: the sequence's, through
// the segments before (after) it.
template <int N, bool REV>
__device__ __forceinline__ float seg_enter(const SelectArgs& a, const SelBlock& sb, int c, int n, float h) {
  const float A2 = a.A[(long)c * N + n] * LOG2E;
  const int m = REV ? sb.nseg - 1 - sb.seg : sb.seg;
#pragma unroll 4
  for (int k = 0; k < m; ++k) {
    const long at = (long)(sb.row0 + (REV ? sb.nseg - 1 - k : k)) * a.D + c;
    h = fmaf(__builtin_amdgcn_exp2f(A2 * a.segdt[at]), h, a.segF[at * N + n]);
  }
  return h;
}

template <typename Tin, int N, int CPL, int L, int W, bool VEC, bool Z>
__global__ __launch_bounds__(64 * W) void k_select_fwd(SelectArgs a, SelectRows q) {
  using S = SelTile<N, CPL>;
  constexpr int LN = S::LN, CG = S::CG, CW = S::CW, NE = S::NE, TL = L / LN, TILE = L * W;
  constexpr int NB = L * N / 64;        // states of a B or C row that a lane loads
  constexpr unsigned EB = sizeof(Tin);
  static_assert(L % LN == 0 && N % NB == 0, "tile");
  struct WaveLds {
    float dt[L][CW], xu[L][CW], B[L][N], C[L][N];
  };
  __shared__ __align__(16) WaveLds lds[W];
  // per chunk: its decay product, and its state from zero, which the owner
  // replaces by the state at its start
  __shared__ __align__(16) float ex[W][2][NE];

  const SelBlock sb = sel_block<CW>(a, q);
  const int lane = lane_id(), w = wave_id_s(), ng = lane / CG, cg = lane % CG;
  const int cl = sb.c0 + cg * CPL, nv = max(0, min(CPL, sb.cend - cl));  // the lane's channels
  const int len = sb.t1;  // the segment's end
  if (sb.seg > 0 && sb.t0 >= len) return;
  WaveLds& my = lds[w];

  // byte offsets of the lane's pieces in a tile's rows
  const unsigned tok = w * L + ng, cb = nv > 0 ? (unsigned)cl * EB : BUF_OOB;
  const unsigned ub = a.u_row * EB, db = a.delta_row * EB, zb = a.z_row * EB, yb = a.D * EB;
  const unsigned uo = tok * ub + cb, dof = tok * db + cb, zo = Z ? tok * zb + cb : 0, yo = tok * yb + cb;
  const int bt = lane * NB / N, bs = lane * NB % N;  // the lane's part of the chunk's B, C
  const unsigned bo = (w * L + bt) * (unsigned)(a.b_row * EB) + (sb.g * N + bs) * EB;
  const unsigned co = (w * L + bt) * (unsigned)(a.c_row * EB) + (sb.g * N + bs) * EB;
  Piece<Tin, CPL, VEC> pu[TL], pd[TL], pz[TL];
  Piece<Tin, NB, VEC> pb, pc;
  const long row0 = sb.tok0 + sb.t0;
  RowsAt tu(a.u, row0, ub), td(a.delta, row0, db), tz(a.z, row0, zb), ty(a.y, row0, yb);
  RowsAt tb(a.Bm, row0, a.b_row * EB), tc(a.Cm, row0, a.c_row * EB);
  auto load = [&](int base) {
    const int rows = min(len - base, TILE);
    const auto ru = tu.rows(rows), rd = td.rows(rows), rb = tb.rows(rows), rc = tc.rows(rows);
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      pu[k].load(ru, uo + k * LN * ub, nv);
      pd[k].load(rd, dof + k * LN * db, nv);
    }
    if constexpr (Z) {
      const auto rz = tz.rows(rows);
#pragma unroll
      for (int k = 0; k < TL; ++k) pz[k].load(rz, zo + k * LN * zb, nv);
    }
    pb.load(rb, bo, NB);
    pc.load(rc, co, NB);
    tu.step(TILE);
    td.step(TILE);
    if constexpr (Z) tz.step(TILE);
    tb.step(TILE);
    tc.step(TILE);
  };
  if (sb.t0 < len) load(sb.t0);

  float A2[CPL][4], h[CPL][4], bias[CPL], skip[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = i < nv ? cl + i : sb.c0;
    bias[i] = or_zero(a.bias, a.A, c);
    skip[i] = or_zero(a.Dskip, a.A, c);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v = a.A[(long)c * N + ng * 4 + j];
      A2[i][j] = i < nv ? v * LOG2E : 0.f;
    }
  }
  // the state that this thread owns, below NE, at the tile's start
  const int own = threadIdx.x;
  int oc, on;
  sel_slot<N, CPL>(own, oc, on);
  const bool has = own < NE && sb.c0 + oc < sb.cend;
  const long oat = ((long)sb.seq * a.D + sb.c0 + oc) * N + on;
  float H = a.h0 && has ? a.h0[oat] : 0.f;
  if (sb.seg > 0 && has) H = seg_enter<N, false>(a, sb, sb.c0 + oc, on, H);
  for (int base = sb.t0; base < len; base += TILE) {
    const int t0 = base + w * L;
    // stage the chunk: dt and dt u per (token, channel), B and C in fp32; past
    // the end dt = 0 and zeros as loaded leave the state as it is
    Piece<Tin, CPL, VEC> cu_[TL], cz[TL];
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      const int tl = ng + LN * k;
      const bool ok = t0 + tl < len;
      float dt[CPL], xu[CPL];
#pragma unroll
      for (int i = 0; i < CPL; ++i) dt[i] = pd[k].get(i) + bias[i];
      if (a.softplus) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) dt[i] = softplus_acc(dt[i]);
      }
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        dt[i] = ok ? dt[i] : 0.f;
        xu[i] = dt[i] * pu[k].get(i);
      }
      lds_put<CPL>(&my.dt[tl][cg * CPL], dt);
      lds_put<CPL>(&my.xu[tl][cg * CPL], xu);
      cu_[k] = pu[k];
      if constexpr (Z) cz[k] = pz[k];
    }
    {
      float v[NB];
#pragma unroll
      for (int e = 0; e < NB; ++e) v[e] = pb.get(e);
      lds_put<NB>(&my.B[bt][bs], v);
#pragma unroll
      for (int e = 0; e < NB; ++e) v[e] = pc.get(e);
      lds_put<NB>(&my.C[bt][bs], v);
    }
    __builtin_amdgcn_wave_barrier();
    if (base + TILE < len) load(base + TILE);

    // first pass: decays, the chunk's state from zero and its part of the outputs
    float dec[L][CPL][4], yp[L * CPL], sdt[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      sdt[i] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) h[i][j] = 0.f;
    }
    const bool live = t0 < len;  // a chunk past the end leaves the state as it is
    if (live) {
#pragma unroll
      for (int t = 0; t < L; ++t) {
        __builtin_amdgcn_sched_barrier(0);
        float dt[CPL], xu[CPL], Bv[4], Cv[4];
        lds_get<CPL>(&my.dt[t][cg * CPL], dt);
        lds_get<CPL>(&my.xu[t][cg * CPL], xu);
        lds_get<4>(&my.B[t][ng * 4], Bv);
        lds_get<4>(&my.C[t][ng * 4], Cv);
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
          sdt[i] += dt[i];
          float s = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            dec[t][i][j] = __builtin_amdgcn_exp2f(dt[i] * A2[i][j]);
            h[i][j] = t == 0 ? xu[i] * Bv[j] : fmaf(dec[t][i][j], h[i][j], xu[i] * Bv[j]);
            s = j == 0 ? Cv[0] * h[i][0] : fmaf(Cv[j], h[i][j], s);
          }
          asm("" : "+v"(s));  // formed here: deferred, every token's states would stay in registers
          yp[t * CPL + i] = s;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      float p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = __builtin_amdgcn_exp2f(sdt[i] * A2[i][j]);
      lds_put<4>(&ex[w][0][(i * 64 + lane) * 4], p);
      lds_put<4>(&ex[w][1][(i * 64 + lane) * 4], h[i]);
    }
    __syncthreads();
    // the states at the chunks' starts, each state by its owner
    if (own < NE) {
      float p[W], f[W];
#pragma unroll
      for (int m = 0; m < W; ++m) {
        p[m] = ex[m][0][own];
        f[m] = ex[m][1][own];
      }
#pragma unroll
      for (int m = 0; m < W; ++m) {
        ex[m][1][own] = H;
        H = fmaf(p[m], H, f[m]);
      }
    }
    __syncthreads();
    const auto ry = ty.rows(min(len - base, TILE));
    ty.step(TILE);
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < CPL; ++i) lds_get<4>(&ex[w][1][(i * 64 + lane) * 4], h[i]);
    if (a.ck && t0 % select_ck(N) == 0) {
      float* ck = a.ck + ((long)(sb.tok0 / select_ck(N) + sb.seq + t0 / select_ck(N)) * a.D + cl) * N + ng * 4;
#pragma unroll
      for (int i = 0; i < CPL; ++i)
        if (i < nv) *reinterpret_cast<float4*>(ck + i * N) = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
    }
    // second pass: what that state adds, decayed, to the outputs
#pragma unroll
    for (int t = 0; t < L; ++t) {
      __builtin_amdgcn_sched_barrier(0);
      float Cv[4];
      lds_get<4>(&my.C[t][ng * 4], Cv);
#pragma unroll
      for (int i = 0; i < CPL; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          h[i][j] *= dec[t][i][j];
          yp[t * CPL + i] = fmaf(Cv[j], h[i][j], yp[t * CPL + i]);
        }
    }
    // sums over the lane groups, LN tokens at a time: lane group ng ends with
    // token ng's, whose u and z it holds
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      float* yk = yp + k * LN * CPL;
      spread_sum<LN * CPL, 5, S::LOW>(yk);
      float y[CPL];
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        y[i] = fmaf(skip[i], cu_[k].get(i), yk[i]);
        if constexpr (Z) {
          const float zv = cz[k].get(i);
          y[i] *= zv * sigmoid_acc(zv);
        }
      }
      store_piece<Tin, CPL, VEC>(ry, yo + k * LN * yb, y, nv);
    }
  }
  if (a.ht && sb.seg == sb.nseg - 1 && has) a.ht[oat] = H;
}

// Backward.  With gy_t = dy_t silu(z_t) and dh_t the gradient of h_t,
//   dh_t = C_t gy_t + a_{t+1} dh_{t+1},   p_t = dh_t a_t h_{t-1},
//   ddt_t = <A, p_t> + u_t <B_t, dh_t>,   dA = sum_t dt_t p_t,   du_t = dt_t <B_t, dh_t> + Dskip gy_t,
//   dB_t = sum_c dh_t dt_t u_t,           dC_t = sum_c gy_t h_t.
// A workgroup walks its sequence's tiles from the last to the first.  The
// states come from the forward's kept ones (one per tile), the
// gradient through the later tiles is carried.  Inside a tile the chunks run
// side by side in both directions as in the forward: each wave forms its decays,
// its state from zero and its gradient from zero, one exchange gives both true
// ends, and a second pass forms the states (kept in registers) and then the
// gradients.  dB and dC of the workgroup's channels go to a partial sum.  Chunks of
// four tokens: decays and states of eight do not fit the registers of twelve waves.
template <typename Tin, int N, int CPL, bool VEC, bool Z>
__global__ __launch_bounds__(16 * select_ck(N)) void k_select_bwd(SelectArgs a, SelectRows q) {
  constexpr int L = 4, W = select_ck(N) / L;
  using S = SelTile<N, CPL>;
  constexpr int LN = S::LN, CG = S::CG, CW = S::CW, NE = S::NE, TL = (L + LN - 1) / LN, TILE = L * W;
  constexpr int NB = L * N / 64 > 0 ? L * N / 64 : 1;
  constexpr unsigned EB = sizeof(Tin);
  static_assert(64 * W >= NE, "an owner for every state");
  struct WaveLds {
    float dt[L][CW], xu[L][CW], gy[L][CW], yp[L][CW], B[L][N], C[L][N];
    float u[L][CW], slope[L][CW], dz[L][CW], odt[L][CW];  // of a lane's own tokens
  };
  __shared__ __align__(16) WaveLds lds[W];
  // per chunk: its decay product, and its state and gradient from zero, which
  // the owner replaces by the state at its start and the gradient at its end
  __shared__ __align__(16) float ex[W][3][NE];

  const SelBlock sb = sel_block<CW>(a, q);
  const int lane = lane_id(), w = wave_id_s(), ng = lane / CG, cg = lane % CG;
  const int cl = sb.c0 + cg * CPL, nv = max(0, min(CPL, sb.cend - cl));
  const int len = sb.t1, tile0 = sb.t0 / TILE;  // the segment's tiles: none past the sequence's end
  const int ntiles = sb.t0 < len ? (len + TILE - 1) / TILE : tile0;
  WaveLds& my = lds[w];

  // the state that this thread owns, below NE: the decayed gradient that enters
  // the tile from the tokens after it, and the kept state at the tile's start
  int oc, on;
  sel_slot<N, CPL>(threadIdx.x, oc, on);
  const bool owner = threadIdx.x < NE, has = owner && sb.c0 + oc < sb.cend;
  const int own = has ? (sb.c0 + oc) * N + on : sb.c0 * N;  // place in a [D, N] state
  float Gc, hk;

  const unsigned tok = w * L + min(ng, L - 1);
  const unsigned cb = nv > 0 && ng < L ? (unsigned)cl * EB : BUF_OOB;
  const unsigned ub = a.u_row * EB, db = a.delta_row * EB, zb = a.z_row * EB, yb = a.D * EB;
  const unsigned uo = tok * ub + cb, dof = tok * db + cb, zo = Z ? tok * zb + cb : 0, yo = tok * yb + cb;
  const int bt = lane * NB / N, bs = lane * NB % N;
  const bool bok = bt < L;
  const unsigned bo = bok ? (w * L + bt) * (unsigned)(a.b_row * EB) + (sb.g * N + bs) * EB : BUF_OOB;
  const unsigned co = bok ? (w * L + bt) * (unsigned)(a.c_row * EB) + (sb.g * N + bs) * EB : BUF_OOB;
  Piece<Tin, CPL, VEC> pu[TL], pd[TL], pz[TL], py[TL];
  Piece<Tin, NB, VEC> pb, pc;
  const long last = sb.tok0 + (long)max(ntiles - 1, 0) * TILE;  // the walk's first tile
  RowsAt tu(a.u, last, ub), td(a.delta, last, db), tz(a.z, last, zb), ty(a.dy, last, yb);
  RowsAt tb(a.Bm, last, a.b_row * EB), tc(a.Cm, last, a.c_row * EB);
  RowsAt tdu(a.du, last, yb), tdd(a.ddelta, last, yb), tdz(a.dz, last, yb);
  RowsAt tbc(a.bcp, (long)sb.blk * a.Ttot + last, 2 * N * 4);
  const float* ck = a.kept + (long)(sb.tok0 / select_ck(N) + sb.seq + max(ntiles - 1, 0)) * a.D * N;
  auto load = [&](int tile) {
    const int rows = min(len - tile * TILE, TILE);
    const auto ru = tu.rows(rows), rd = td.rows(rows), rb = tb.rows(rows), rc = tc.rows(rows);
    const auto ry = ty.rows(rows);
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      pu[k].load(ru, uo + k * LN * ub, nv);
      pd[k].load(rd, dof + k * LN * db, nv);
      py[k].load(ry, yo + k * LN * yb, nv);
    }
    if constexpr (Z) {
      const auto rz = tz.rows(rows);
#pragma unroll
      for (int k = 0; k < TL; ++k) pz[k].load(rz, zo + k * LN * zb, nv);
    }
    pb.load(rb, bo, NB);
    pc.load(rc, co, NB);
    hk = ck[own];
    tu.step(-TILE);
    td.step(-TILE);
    if constexpr (Z) tz.step(-TILE);
    ty.step(-TILE);
    tb.step(-TILE);
    tc.step(-TILE);
    ck -= (long)a.D * N;
  };
  if (ntiles > tile0) load(ntiles - 1);

  float A2[CPL][4], dA[CPL][4], bias[CPL], skip[CPL], dD[CPL], dbias[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = i < nv ? cl + i : sb.c0;
    bias[i] = or_zero(a.bias, a.A, c);
    skip[i] = or_zero(a.Dskip, a.A, c);
    dD[i] = dbias[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v = a.A[(long)c * N + ng * 4 + j];
      A2[i][j] = i < nv ? v * LOG2E : 0.f;
      dA[i][j] = 0.f;
    }
  }
  Gc = a.dht && has ? a.dht[(long)sb.seq * a.D * N + own] : 0.f;
  if (sb.seg < sb.nseg - 1 && has) Gc = seg_enter<N, true>(a, sb, sb.c0 + oc, on, Gc);
  for (int tile = ntiles - 1; tile >= tile0; --tile) {
    const int base = tile * TILE, t0 = base + w * L;
    float h[CPL][4], G[CPL][4];
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      const int tl = ng + LN * k;
      const bool ok = tl < L && t0 + tl < len;
      float dt[CPL], xu[CPL], gy[CPL], uv[CPL], sl[CPL], dz[CPL];
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        dt[i] = pd[k].get(i) + bias[i];
        sl[i] = 1.f;
        uv[i] = pu[k].get(i);
        gy[i] = py[k].get(i);
      }
      if (a.softplus) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
          sl[i] = sigmoid_acc(dt[i]);
          dt[i] = softplus_acc(dt[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        dt[i] = ok ? dt[i] : 0.f;
        xu[i] = dt[i] * uv[i];
        if constexpr (Z) {
          const float zv = pz[k].get(i), sg = sigmoid_acc(zv);
          dz[i] = gy[i] * sg * fmaf(zv, 1.f - sg, 1.f);
          gy[i] *= zv * sg;
        }
      }
      if (tl < L) {
        lds_put<CPL>(&my.dt[tl][cg * CPL], dt);
        lds_put<CPL>(&my.xu[tl][cg * CPL], xu);
        lds_put<CPL>(&my.gy[tl][cg * CPL], gy);
        lds_put<CPL>(&my.u[tl][cg * CPL], uv);
        lds_put<CPL>(&my.odt[tl][cg * CPL], dt);
        lds_put<CPL>(&my.slope[tl][cg * CPL], sl);
        if constexpr (Z) lds_put<CPL>(&my.dz[tl][cg * CPL], dz);
      }
    }
    if (bok) {
      float v[NB];
#pragma unroll
      for (int e = 0; e < NB; ++e) v[e] = pb.get(e);
      lds_put<NB>(&my.B[bt][bs], v);
#pragma unroll
      for (int e = 0; e < NB; ++e) v[e] = pc.get(e);
      lds_put<NB>(&my.C[bt][bs], v);
    }
    const float hs0 = hk;
    __builtin_amdgcn_wave_barrier();
    if (tile > tile0) load(tile - 1);

    // the chunk from zero, forward then backward
    float dec[L][CPL][4], sdt[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) sdt[i] = 0.f;
#pragma unroll
    for (int t = 0; t < L; ++t) {
      __builtin_amdgcn_sched_barrier(0);
      float dt[CPL], xu[CPL], Bv[4];
      lds_get<CPL>(&my.dt[t][cg * CPL], dt);
      lds_get<CPL>(&my.xu[t][cg * CPL], xu);
      lds_get<4>(&my.B[t][ng * 4], Bv);
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        sdt[i] += dt[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          dec[t][i][j] = __builtin_amdgcn_exp2f(dt[i] * A2[i][j]);
          h[i][j] = t == 0 ? xu[i] * Bv[j] : fmaf(dec[t][i][j], h[i][j], xu[i] * Bv[j]);
        }
      }
    }
#pragma unroll
    for (int t = L - 1; t >= 0; --t) {
      __builtin_amdgcn_sched_barrier(0);
      float gy[CPL], Cv[4];
      lds_get<CPL>(&my.gy[t][cg * CPL], gy);
      lds_get<4>(&my.C[t][ng * 4], Cv);
#pragma unroll
      for (int i = 0; i < CPL; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          G[i][j] = dec[t][i][j] * (t == L - 1 ? Cv[j] * gy[i] : fmaf(Cv[j], gy[i], G[i][j]));
    }
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      float p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = __builtin_amdgcn_exp2f(sdt[i] * A2[i][j]);
      lds_put<4>(&ex[w][0][(i * 64 + lane) * 4], p);
      lds_put<4>(&ex[w][1][(i * 64 + lane) * 4], h[i]);
      lds_put<4>(&ex[w][2][(i * 64 + lane) * 4], G[i]);
    }
    __syncthreads();
    if (owner) {
      const int s = threadIdx.x;
      float p[W], f[W], q[W], c = hs0;
#pragma unroll
      for (int m = 0; m < W; ++m) {
        p[m] = ex[m][0][s];
        f[m] = ex[m][1][s];
        q[m] = ex[m][2][s];
      }
#pragma unroll
      for (int m = 0; m < W; ++m) {
        ex[m][1][s] = c;
        c = fmaf(p[m], c, f[m]);
      }
#pragma unroll
      for (int m = W - 1; m >= 0; --m) {
        ex[m][2][s] = Gc;
        Gc = fmaf(p[m], Gc, q[m]);
      }
    }
    __syncthreads();
    // second pass: the states (hs[t] enters token t)
    float hs[L + 1][CPL][4];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      lds_get<4>(&ex[w][1][(i * 64 + lane) * 4], hs[0][i]);
      lds_get<4>(&ex[w][2][(i * 64 + lane) * 4], G[i]);
    }
#pragma unroll
    for (int t2 = 0; t2 < L; t2 += 2) {
      float s[2 * CPL];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        __builtin_amdgcn_sched_barrier(0);
        const int t = t2 + tt;
        float xu[CPL], Bv[4], Cv[4];
        lds_get<CPL>(&my.xu[t][cg * CPL], xu);
        lds_get<4>(&my.B[t][ng * 4], Bv);
        if constexpr (Z) lds_get<4>(&my.C[t][ng * 4], Cv);
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
          float v = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            hs[t + 1][i][j] = fmaf(dec[t][i][j], hs[t][i][j], xu[i] * Bv[j]);
            if constexpr (Z) v = j == 0 ? Cv[0] * hs[t + 1][i][0] : fmaf(Cv[j], hs[t + 1][i][j], v);
          }
          s[tt * CPL + i] = v;
        }
      }
      if constexpr (Z) {  // the ungated output, for dz
        constexpr int VL = 2 * CPL / LN > 0 ? 2 * CPL / LN : 1;
        spread_sum<2 * CPL, 5, S::LOW>(s);
        const int v = LN >= 2 * CPL ? ng / (LN / (2 * CPL) > 0 ? LN / (2 * CPL) : 1) : ng * VL;
        float o[VL];
#pragma unroll
        for (int i = 0; i < VL; ++i) o[i] = s[i];
        lds_put<VL>(&my.yp[t2 + v / CPL][cg * CPL + v % CPL], o);
      }
    }
    // second pass: the gradients
    const int rows = min(len - base, TILE);
    const auto rbc = tbc.rows(rows);
#pragma unroll
    for (int t2 = L - 2; t2 >= 0; t2 -= 2) {
      float bc[16];
#pragma unroll
      for (int tt = 1; tt >= 0; --tt) {
        __builtin_amdgcn_sched_barrier(0);
        const int t = t2 + tt;
        float dt[CPL], xu[CPL], gy[CPL], Bv[4], Cv[4], sm[2 * CPL];
        lds_get<CPL>(&my.dt[t][cg * CPL], dt);
        lds_get<CPL>(&my.xu[t][cg * CPL], xu);
        lds_get<CPL>(&my.gy[t][cg * CPL], gy);
        lds_get<4>(&my.B[t][ng * 4], Bv);
        lds_get<4>(&my.C[t][ng * 4], Cv);
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float dh = fmaf(Cv[j], gy[i], G[i][j]);
            G[i][j] = dec[t][i][j] * dh;
            const float p = G[i][j] * hs[t][i][j];
            sm[i] = j == 0 ? dh * Bv[0] : fmaf(dh, Bv[j], sm[i]);
            sm[CPL + i] = j == 0 ? A2[i][0] * p : fmaf(A2[i][j], p, sm[CPL + i]);
            dA[i][j] = fmaf(dt[i], p, dA[i][j]);
            bc[tt * 8 + j] = i == 0 ? dh * xu[0] : fmaf(dh, xu[i], bc[tt * 8 + j]);
            bc[tt * 8 + 4 + j] = i == 0 ? gy[0] * hs[t + 1][0][j] : fmaf(gy[i], hs[t + 1][i][j], bc[tt * 8 + 4 + j]);
          }
        }
        // over the states: <B, dh> and <A, p> replace the token's xu and dt
        constexpr int VL = 2 * CPL / LN > 0 ? 2 * CPL / LN : 1;
        spread_sum<2 * CPL, 5, S::LOW>(sm);
        const int v = LN >= 2 * CPL ? ng / (LN / (2 * CPL) > 0 ? LN / (2 * CPL) : 1) : ng * VL;
        float o[VL];
#pragma unroll
        for (int i = 0; i < VL; ++i) o[i] = sm[i];
        __builtin_amdgcn_wave_barrier();
        lds_put<VL>(v < CPL ? &my.xu[t][cg * CPL + v] : &my.dt[t][cg * CPL + v - CPL], o);
      }
      // over the channels, two tokens' 16 values; dB and dC of a token side by side
      constexpr int VB = 16 / CG > 0 ? 16 / CG : 1, REST = CG / 16 > 0 ? CG / 16 : 1;
      spread_sum<16, S::LOW - 1, 0>(bc);
      const int v = CG >= 16 ? cg / REST : cg * VB;
      const unsigned at = ((w * L + t2 + (v >> 3)) * 2 * N + ((v >> 2) & 1) * N + ng * 4 + (v & 3)) * 4;
#pragma unroll
      for (int i = 0; i < VB; ++i)
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(bc[i]), rbc, cg % REST ? BUF_OOB : at + 4 * i, 0, 0);
    }
    __builtin_amdgcn_wave_barrier();
    // the own tokens' gradients
    const auto rdu = tdu.rows(rows), rdd = tdd.rows(rows), rdz = tdz.rows(Z ? rows : 0);
    tbc.step(-TILE);
    tdu.step(-TILE);
    tdd.step(-TILE);
    if constexpr (Z) tdz.step(-TILE);
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      const int tl = min(ng + LN * k, L - 1);
      const bool ok = ng + LN * k < L && t0 + tl < len;
      float sbv[CPL], sa[CPL], yp[CPL], du[CPL], dd[CPL], dz[CPL], uv[CPL], sl[CPL], gy[CPL], dt[CPL];
      lds_get<CPL>(&my.odt[tl][cg * CPL], dt);
      lds_get<CPL>(&my.xu[tl][cg * CPL], sbv);
      lds_get<CPL>(&my.dt[tl][cg * CPL], sa);
      lds_get<CPL>(&my.u[tl][cg * CPL], uv);
      lds_get<CPL>(&my.gy[tl][cg * CPL], gy);
      lds_get<CPL>(&my.slope[tl][cg * CPL], sl);
      if constexpr (Z) {
        lds_get<CPL>(&my.yp[tl][cg * CPL], yp);
        lds_get<CPL>(&my.dz[tl][cg * CPL], dz);
      }
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        du[i] = fmaf(dt[i], sbv[i], skip[i] * gy[i]);
        dd[i] = fmaf(uv[i], sbv[i], LN2 * sa[i]) * sl[i];
        dD[i] = fmaf(gy[i], uv[i], dD[i]);
        dbias[i] += ok ? dd[i] : 0.f;
        if constexpr (Z) dz[i] *= fmaf(skip[i], uv[i], yp[i]);
      }
      store_piece<Tin, CPL, VEC>(rdu, yo + k * LN * yb, du, nv);
      store_piece<Tin, CPL, VEC>(rdd, yo + k * LN * yb, dd, nv);
      if constexpr (Z) store_piece<Tin, CPL, VEC>(rdz, yo + k * LN * yb, dz, nv);
    }
  }
  // the sequence's parameter gradients: the waves' sums in order, dD and dbias
  // also over the lane groups, which held different tokens
  __syncthreads();
  float* red = &ex[0][1][0];  // [W][2][CPL][64], in the chunks' second parts
  static_assert(2 * CPL * 64 <= NE, "room for the sums");
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    lds_put<4>(&ex[w][0][(i * 64 + lane) * 4], dA[i]);
    red[w * 3 * NE + (0 * CPL + i) * 64 + lane] = dD[i];
    red[w * 3 * NE + (1 * CPL + i) * 64 + lane] = dbias[i];
  }
  __syncthreads();
  const long part = (long)(sb.row0 + sb.seg) * a.D;
  if (has) {
    float v = ex[0][0][threadIdx.x];
#pragma unroll
    for (int m = 1; m < W; ++m) v += ex[m][0][threadIdx.x];
    a.dap[(part + sb.c0 + oc) * (N + 2) + on] = v;
    if (a.dh0 && sb.seg == 0) a.dh0[(long)sb.seq * a.D * N + own] = Gc;
  }
  const int ch = threadIdx.x % CW, which = threadIdx.x / CW;
  if (which < 2 && sb.c0 + ch < sb.cend) {
    float v = 0.f;
    for (int m = 0; m < W; ++m)
      for (int e = 0; e < min(LN, L); ++e)
        v += red[m * 3 * NE + (which * CPL + ch % CPL) * 64 + e * CG + ch / CPL];
    a.dap[(part + sb.c0 + ch) * (N + 2) + N + which] = v;
  }
}

// The sums after the main kernel, in one launch: the first `nbc` workgroups add dB
// and dC of every (token, group, state) over the channel blocks, four values a
// thread, the others dA, dD and dbias over the segments; both in order.
template <typename Tin>
__global__ __launch_bounds__(256) void k_select_sums(SelectArgs a, int rows, int nbc) {
  if ((int)blockIdx.x >= nbc) {
    const int w = a.N + 2;
    const long n = (long)a.D * w, e = (long)(blockIdx.x - nbc) * 256 + threadIdx.x;
    if (e >= n) return;
    float sum = 0.f;
#pragma unroll 4
    for (int s = 0; s < rows; ++s) sum += a.dap[s * n + e];
    const int k = e % w;
    const long c = e / w;
    if (k < a.N) a.dA[c * a.N + k] = sum;
    else if (k == a.N) { if (a.dD) a.dD[c] = sum; }
    else if (a.dbias) a.dbias[c] = sum;
    return;
  }
  const int N2 = 2 * a.N;
  const long n = (long)a.Ttot * a.G * N2;
  const long e = ((long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (e >= n) return;
  const int s = e % N2;
  const long tg = e / N2;
  const int g = tg / a.Ttot;
  const long t = tg % a.Ttot;
  const float4* p = reinterpret_cast<const float4*>(a.bcp + ((long)g * a.nblk * a.Ttot + t) * N2 + s);
  const long row = (long)a.Ttot * N2 / 4;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int b = 0; b < a.nblk; ++b) {
    const float4 f = p[b * row];
    v = make_float4(v.x + f.x, v.y + f.y, v.z + f.z, v.w + f.w);
  }
  Tin* out = static_cast<Tin*>(s < a.N ? a.dB : a.dC) + (t * a.G + g) * a.N + (s < a.N ? s : s - a.N);
  store_elem(out, v.x);
  store_elem(out + 1, v.y);
  store_elem(out + 2, v.z);
  store_elem(out + 3, v.w);
}

// One token per row: a lane holds 4 states of one channel, consecutive lanes
// consecutive states, so that a wave reads and writes whole kilobytes of the
// state.  A thread takes R rows, all loaded before the first is used.  200 rows of
// 4,096 channels x 16 states: 20.8 us for 105 MB of states and 5 MB beside (5.3
// TB/s, partly from the on-die cache); one row of 2,048: 2.5 us.
template <typename Tin, int N, bool VEC, int R>
__global__ __launch_bounds__(256) void k_select_step(SelectArgs a) {
  constexpr int LN = N / 4;
  const int nbx = (a.D * LN + 255) / 256;  // workgroups per R rows
  const int rb = blockIdx.x / nbx, e = (blockIdx.x - rb * nbx) * 256 + threadIdx.x;
  const int c = e / LN, ng = e % LN;
  const bool on = c < a.D;  // whole lane groups: a channel's lanes agree
  const int cc = on ? c : a.D - 1, g = cc / (a.D / a.G);
  int row[R], slot[R];
  bool live[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    row[r] = min(rb * R + r, a.S - 1);
    slot[r] = a.slots ? a.slots[row[r]] : row[r];
    live[r] = slot[r] >= 0 && slot[r] < a.num_slots;  // else padding
  }
  // every load unconditional (a load under a branch is waited for on the spot):
  // padding reads slot 0, or without any slot an A row, and drops it; without z, u
  const bool any = a.num_slots > 0;
  const Tin* zp = static_cast<const Tin*>(a.z ? a.z : a.u);
  const long zrow = a.z ? a.z_row : a.u_row;
  float A2[4], hv[R][4];
  Piece<Tin, 4, VEC> pb[R], pc[R];
  Piece<Tin, 1, true> pu[R], pd[R], pz[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float* hp = (any ? a.state : a.A) + ((long)(live[r] ? slot[r] : 0) * a.D + cc) * N + ng * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) hv[r][j] = __builtin_nontemporal_load(hp + j);
    pu[r].load(static_cast<const Tin*>(a.u) + row[r] * a.u_row + cc, 1);
    pd[r].load(static_cast<const Tin*>(a.delta) + row[r] * a.delta_row + cc, 1);
    pz[r].load(zp + row[r] * zrow + cc, 1);
    pb[r].load(static_cast<const Tin*>(a.Bm) + row[r] * a.b_row + g * N + ng * 4, 4);
    pc[r].load(static_cast<const Tin*>(a.Cm) + row[r] * a.c_row + g * N + ng * 4, 4);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) A2[j] = a.A[(long)cc * N + ng * 4 + j] * LOG2E;
  const float bias = a.bias ? a.bias[cc] : 0.f, skip = a.Dskip ? a.Dskip[cc] : 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float uv = pu[r].get(0), raw = pd[r].get(0) + bias;
    const float dt = a.softplus ? softplus_acc(raw) : raw, xu = dt * uv;
    float h[4], s = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      h[j] = fmaf(__builtin_amdgcn_exp2f(dt * A2[j]), hv[r][j], xu * pb[r].get(j));
      s = fmaf(pc[r].get(j), h[j], s);
    }
    s = xsum<0>(s);
    if constexpr (LN >= 4) s = xsum<1>(s);
    if constexpr (LN >= 8) s = xsum<2>(s);
    const bool mine = on && rb * R + r < a.S;
    if (mine && live[r]) {
      float* hp = a.state + ((long)slot[r] * a.D + cc) * N + ng * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) __builtin_nontemporal_store(h[j], hp + j);
    }
    if (mine && ng == 0) {
      float v = fmaf(skip, uv, s);
      if (a.z) {
        const float zv = pz[r].get(0);
        v *= zv * sigmoid_acc(zv);
      }
      store_elem(static_cast<Tin*>(a.y) + (long)row[r] * a.D + c, live[r] ? v : 0.f);
    }
  }
}

// Whether every piece of C channels, and of nb states of a B or C row, is loaded and
// stored at once, or value by value (4 x 4,096 tokens, 4,096 channels, 16 states: 363 /
// 462 us forward, 954 / 1,033 backward).
static bool rows_vec(const SelectArgs& a, int C, int nb, bool bwd) {
  const long eb = a.bf16 ? 2 : 4;
  auto ok = [&](const void* p, long row, long n) { return !p || ((uintptr_t)p % (n * eb) == 0 && row % n == 0); };
  const bool v = (a.D / a.G) % C == 0 && ok(a.u, a.u_row, C) && ok(a.delta, a.delta_row, C) &&
                 ok(a.z, a.z_row, C) && ok(a.Bm, a.b_row, nb) && ok(a.Cm, a.c_row, nb);
  if (!bwd) return v && ok(a.y, a.D, C);
  return v && ok(a.dy, a.D, C) && ok(a.du, a.D, C) && ok(a.ddelta, a.D, C) && ok(a.dz, a.D, C);
}

template <typename Tin, int N, bool REV>
static void run_seg(const SelectArgs& a, const SelectRows& q, unsigned grid) {
  if (a.segs <= 1) return;
  if (rows_vec(a, SEL_CPL, N / 8, REV)) k_select_seg<Tin, N, SEL_CPL, true, REV><<<grid, 64 * sel_waves(N), 0, a.stream>>>(a, q);
  else k_select_seg<Tin, N, SEL_CPL, false, REV><<<grid, 64 * sel_waves(N), 0, a.stream>>>(a, q);
}

template <typename Tin, int N>
static hipError_t run_fwd(const SelectArgs& a, const SelectRows& q) {
  constexpr int CPL = SEL_CPL, L = 8, W = sel_waves(N);
  static_assert(SelTile<N, CPL>::CW == select_block_channels(N), "one block of channels throughout");
  const unsigned grid = (unsigned)q.rows * a.G * a.nblk;
  run_seg<Tin, N, false>(a, q, grid);
  const bool vec = rows_vec(a, CPL, L * N / 64, false);
  if (vec && a.z) k_select_fwd<Tin, N, CPL, L, W, true, true><<<grid, 64 * W, 0, a.stream>>>(a, q);
  else if (vec) k_select_fwd<Tin, N, CPL, L, W, true, false><<<grid, 64 * W, 0, a.stream>>>(a, q);
  else if (a.z) k_select_fwd<Tin, N, CPL, L, W, false, true><<<grid, 64 * W, 0, a.stream>>>(a, q);
  else k_select_fwd<Tin, N, CPL, L, W, false, false><<<grid, 64 * W, 0, a.stream>>>(a, q);
  return hipGetLastError();
}

template <typename Tin, int N>
static hipError_t run_bwd(const SelectArgs& a, const SelectRows& q) {
  constexpr int CPL = SEL_CPL;
  const unsigned grid = (unsigned)q.rows * a.G * a.nblk;
  if (grid > 0) {
    run_seg<Tin, N, true>(a, q, grid);
    const bool vec = rows_vec(a, CPL, N >= 16 ? N / 16 : 1, true);
    if (vec && a.z) k_select_bwd<Tin, N, CPL, true, true><<<grid, 16 * select_ck(N), 0, a.stream>>>(a, q);
    else if (vec) k_select_bwd<Tin, N, CPL, true, false><<<grid, 16 * select_ck(N), 0, a.stream>>>(a, q);
    else if (a.z) k_select_bwd<Tin, N, CPL, false, true><<<grid, 16 * select_ck(N), 0, a.stream>>>(a, q);
    else k_select_bwd<Tin, N, CPL, false, false><<<grid, 16 * select_ck(N), 0, a.stream>>>(a, q);
  }
  const long nbc = ((long)a.Ttot * a.G * 2 * N / 4 + 255) / 256, np = ((long)a.D * (N + 2) + 255) / 256;
  if (nbc + np > INT32_MAX) return hipErrorInvalidValue;
  k_select_sums<Tin><<<(unsigned)(nbc + np), 256, 0, a.stream>>>(a, q.rows, (int)nbc);
  return hipGetLastError();
}

template <typename Tin, int N, int R>
static hipError_t step_rows(const SelectArgs& a) {
  const long grid = ((long)a.D * (N / 4) + 255) / 256 * ((a.S + R - 1) / R);
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  const long m = 4 * sizeof(Tin);
  const bool vec = (uintptr_t)a.Bm % m == 0 && (uintptr_t)a.Cm % m == 0 && a.b_row % 4 == 0 && a.c_row % 4 == 0;
  if (vec) k_select_step<Tin, N, true, R><<<(unsigned)grid, 256, 0, a.stream>>>(a);
  else k_select_step<Tin, N, false, R><<<(unsigned)grid, 256, 0, a.stream>>>(a);
  return hipGetLastError();
}
template <typename Tin, int N>
static hipError_t run_step(const SelectArgs& a) {
  // four rows a thread where that leaves four workgroups per CU (16 states, us with
  // one / four rows: 8 x 4,096 channels 2.8 / 3.5; 64 x 4,096 7.7 / 6.6; 200 x 4,096
  // 21.2 / 20.8; 512 x 2,048 27.5 / 26.1)
  return (long)a.S * a.D * (N / 4) >= 4L * 1024 * 256 ? step_rows<Tin, N, 4>(a) : step_rows<Tin, N, 1>(a);
}

#define SELECT_DISPATCH(fn, ...)                                                                       \
  (a.N == 8    ? (a.bf16 ? fn<bf16_t, 8>(__VA_ARGS__) : fn<float, 8>(__VA_ARGS__))                     \
   : a.N == 16 ? (a.bf16 ? fn<bf16_t, 16>(__VA_ARGS__) : fn<float, 16>(__VA_ARGS__))                   \
   : a.N == 32 ? (a.bf16 ? fn<bf16_t, 32>(__VA_ARGS__) : fn<float, 32>(__VA_ARGS__)) : hipErrorInvalidValue)

hipError_t launch_select_fwd(const SelectArgs& a, const SelectRows& q) {
  return a.S == 0 ? hipSuccess : SELECT_DISPATCH(run_fwd, a, q);
}
hipError_t launch_select_bwd(const SelectArgs& a, const SelectRows& q) { return SELECT_DISPATCH(run_bwd, a, q); }
hipError_t launch_select_step(const SelectArgs& a) {
  return a.S == 0 ? hipSuccess : SELECT_DISPATCH(run_step, a);
}

}  // namespace comba
