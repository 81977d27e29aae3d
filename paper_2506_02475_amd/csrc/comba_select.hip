// Selective state space scan: per channel c and state n
//
//   h_t = exp(dt_t A) h_{t-1} + dt_t u_t B_t,   s_t = <C_t, h_t> + Dskip u_t,   y_t = s_t silu(z_t)
//
// A decay of its own for every (channel, state, token) leaves nothing for the
// matrix units: the work is one exponential and four vector operations per
// (channel, state, token), and these, not the bytes, bound every long call.
//
// Layout of a wave: CW channels x N states.  A lane holds CPL channels x 4
// states (lane group ng = lane / CG takes states 4 ng .. 4 ng + 3, lane cg = lane
// % CG takes channels CPL cg ..), so that sums over states are three in-lane
// adds and log2(N / 4) lane exchanges for CPL channels at once, and sums over
// channels (the gradients of B and C) start with in-lane adds as well.
//
// Time: a workgroup's W waves take consecutive chunks of L tokens of a tile.  A
// wave forms its chunk's decays once and keeps them in registers, with the
// chunk's state from a zero start; the chunks' (product of decays, state) pairs
// are combined through LDS, and a second pass, now from the true state, reuses
// the decays.  The second pass costs three operations more per value than a
// walk token by token, but leaves W times as many waves.
#include "comba_layer_device.hpp"
#include "comba_layer_launch.h"

namespace comba {

template <int N, int CPL>
struct SelTile {
  static constexpr int LN = N / 4;     // lane groups over the states
  static constexpr int CG = 64 / LN;   // lanes over the channels
  static constexpr int CW = CG * CPL;  // channels of a wave
  static constexpr int LNB = LN == 2 ? 1 : LN == 4 ? 2 : 3;  // log2
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

// B or C rows of a chunk as loaded: lane l takes NB consecutive states of one token.
template <typename Tin, int N, int L>
struct StateRows {
  static constexpr int NB = L * N / 64;
  static_assert(NB >= 1 && N % NB == 0, "a lane's states lie in one token");
  float v[NB];
  __device__ __forceinline__ static int token() { return lane_id() * NB / N; }
  __device__ __forceinline__ static int state() { return lane_id() * NB % N; }
  __device__ __forceinline__ void load(const Tin* p) {
#pragma unroll
    for (int e = 0; e < NB; ++e) v[e] = to_f(p[e]);
  }
};

template <typename Tin, int N, int CPL, int L, int W, bool VEC>
__global__ __launch_bounds__(64 * W) void k_select_fwd(SelectArgs a) {
  using S = SelTile<N, CPL>;
  constexpr int LN = S::LN, CG = S::CG, CW = S::CW, TL = L / LN, TILE = L * W;
  static_assert(L % LN == 0, "tokens per lane");
  using SR = StateRows<Tin, N, L>;
  struct WaveLds {
    float dt[L][CW], xu[L][CW], B[L][N], C[L][N];
  };
  __shared__ __align__(16) WaveLds lds[W];
  __shared__ float4 ex[W - 1][2][CPL][64];  // a chunk's decay product and its state from zero
  __shared__ float4 hb[CPL][64];            // the state at the tile's start

  const int lane = lane_id(), w = wave_id_s(), ng = lane / CG, cg = lane % CG;
  const int Dg = a.D / a.G, nblk = (Dg + CW - 1) / CW, nb = a.G * nblk;
  const int seq = blockIdx.x / nb, blk = blockIdx.x % nb, g = blk / nblk;
  const int cl = g * Dg + (blk % nblk) * CW + cg * CPL;  // first channel of the lane
  const int nv = max(0, min(CPL, (g + 1) * Dg - cl));    // how many of them exist
  const int cs = nv > 0 ? cl : g * Dg, ns = max(nv, 1);   // a place that may be read
  int tok0, tok1;
  seq_range(a.cu_seqlens, seq, a.Tseq, a.Ttot, tok0, tok1);
  const int len = tok1 - tok0;
  WaveLds& my = lds[w];

  float A2[CPL][4], h[CPL][4], bias[CPL], skip[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = min(cs + i, cs + ns - 1);
    bias[i] = a.bias ? a.bias[c] : 0.f;
    skip[i] = a.Dskip ? a.Dskip[c] : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      A2[i][j] = i < nv ? a.A[(long)c * N + ng * 4 + j] * LOG2E : 0.f;
      h[i][j] = a.h0 ? a.h0[((long)seq * a.D + c) * N + ng * 4 + j] : 0.f;
    }
  }
  if (w == W - 1) {
#pragma unroll
    for (int i = 0; i < CPL; ++i) hb[i][lane] = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
  }

  Piece<Tin, CPL, VEC> pu[TL], pd[TL], pz[TL];
  SR pb, pc;
  const Tin *u = static_cast<const Tin*>(a.u), *delta = static_cast<const Tin*>(a.delta),
            *z = static_cast<const Tin*>(a.z), *Bm = static_cast<const Tin*>(a.Bm),
            *Cm = static_cast<const Tin*>(a.Cm);
  // a chunk's rows; past the end the last row, whose values staging drops
  auto load = [&](int t0) {
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      const long row = tok0 + min(t0 + ng + LN * k, len - 1);
      pu[k].load(u + row * a.u_row + cs, ns);
      pd[k].load(delta + row * a.delta_row + cs, ns);
      if (z) pz[k].load(z + row * a.z_row + cs, ns);
    }
    const long row = tok0 + min(t0 + SR::token(), len - 1);
    pb.load(Bm + row * a.b_row + g * N + SR::state());
    pc.load(Cm + row * a.c_row + g * N + SR::state());
  };
  if (len > 0) load(w * L);
  for (int base = 0; base < len; base += TILE) {
    const int t0 = base + w * L;
    // stage the chunk: dt and dt u per (token, channel), B and C in fp32; zeros
    // past the end, which leave the state as it is
    Piece<Tin, CPL, VEC> cu_[TL], cz[TL];
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      const int tl = ng + LN * k;
      const bool ok = t0 + tl < len;
      float dt[CPL], xu[CPL];
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        const float raw = pd[k].get(i) + bias[i];
        const float d = a.softplus ? softplus_acc(raw) : raw;
        const bool on = ok && i < nv;
        dt[i] = on ? d : 0.f;
        xu[i] = on ? d * pu[k].get(i) : 0.f;
      }
      lds_put<CPL>(&my.dt[tl][cg * CPL], dt);
      lds_put<CPL>(&my.xu[tl][cg * CPL], xu);
      cu_[k] = pu[k];
      cz[k] = pz[k];
    }
    {
      const int tl = SR::token();
      const bool ok = t0 + tl < len;
#pragma unroll
      for (int e = 0; e < SR::NB; ++e) {
        my.B[tl][SR::state() + e] = ok ? pb.v[e] : 0.f;
        my.C[tl][SR::state() + e] = ok ? pc.v[e] : 0.f;
      }
    }
    __builtin_amdgcn_wave_barrier();
    if (base + TILE < len) load(t0 + TILE);

    // first pass: decays, the chunk's state from zero
    float dec[L][CPL][4], sdt[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      sdt[i] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) h[i][j] = 0.f;
    }
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
          h[i][j] = fmaf(dec[t][i][j], h[i][j], xu[i] * Bv[j]);
        }
      }
    }
    if (w < W - 1) {
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        ex[w][0][i][lane] = make_float4(
            __builtin_amdgcn_exp2f(sdt[i] * A2[i][0]), __builtin_amdgcn_exp2f(sdt[i] * A2[i][1]),
            __builtin_amdgcn_exp2f(sdt[i] * A2[i][2]), __builtin_amdgcn_exp2f(sdt[i] * A2[i][3]));
        ex[w][1][i][lane] = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
      }
    }
    __syncthreads();
    // the true state at the chunk's start: the tile's, through the chunks before
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const float4 f = hb[i][lane];
      h[i][0] = f.x;
      h[i][1] = f.y;
      h[i][2] = f.z;
      h[i][3] = f.w;
    }
    for (int m = 0; m < w; ++m) {
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        const float4 p = ex[m][0][i][lane], f = ex[m][1][i][lane];
        h[i][0] = fmaf(p.x, h[i][0], f.x);
        h[i][1] = fmaf(p.y, h[i][1], f.y);
        h[i][2] = fmaf(p.z, h[i][2], f.z);
        h[i][3] = fmaf(p.w, h[i][3], f.w);
      }
    }
    __syncthreads();
    if (a.ck && t0 % SELECT_CK == 0 && t0 < len) {
      float* ck = a.ck + ((long)(tok0 / SELECT_CK + seq + t0 / SELECT_CK) * a.D + cl) * N + ng * 4;
#pragma unroll
      for (int i = 0; i < CPL; ++i)
        if (i < nv) *reinterpret_cast<float4*>(ck + i * N) = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
    }
    // second pass: the states, and their sums with C, LN tokens at a time: lane
    // group ng ends with token ng's, whose u and z it holds
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      float yp[LN * CPL];
#pragma unroll
      for (int e = 0; e < LN; ++e) {
        const int t = k * LN + e;
        __builtin_amdgcn_sched_barrier(0);
        float xu[CPL], Bv[4], Cv[4];
        lds_get<CPL>(&my.xu[t][cg * CPL], xu);
        lds_get<4>(&my.B[t][ng * 4], Bv);
        lds_get<4>(&my.C[t][ng * 4], Cv);
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
          float s = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            h[i][j] = fmaf(dec[t][i][j], h[i][j], xu[i] * Bv[j]);
            s = j == 0 ? Cv[0] * h[i][0] : fmaf(Cv[j], h[i][j], s);
          }
          yp[e * CPL + i] = s;
        }
      }
      spread_sum<LN * CPL, 5, 6 - S::LNB>(yp);
      const int t = t0 + ng + LN * k;
      if (t < len) {
        float y[CPL];
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
          y[i] = fmaf(skip[i], cu_[k].get(i), yp[i]);
          if (z) {
            const float zv = cz[k].get(i);
            y[i] *= zv * sigmoid_acc(zv);
          }
        }
        store_piece<Tin, CPL, VEC>(static_cast<Tin*>(a.y) + (long)(tok0 + t) * a.D + cl, y, nv);
      }
    }
    if (w == W - 1) {
#pragma unroll
      for (int i = 0; i < CPL; ++i) hb[i][lane] = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
    }
  }
  if (a.ht && w == W - 1) {
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i < nv) a.ht[((long)seq * a.D + cl + i) * N + ng * 4 + j] = h[i][j];
  }
}

// Backward.  With gy_t = dy_t silu(z_t) and dh_t the gradient of h_t,
//   dh_t = C_t gy_t + a_{t+1} dh_{t+1},   p_t = dh_t a_t h_{t-1},
//   ddt_t = <A, p_t> + u_t <B_t, dh_t>,   dA = sum_t dt_t p_t,   du_t = dt_t <B_t, dh_t> + Dskip gy_t,
//   dB_t = sum_c dh_t dt_t u_t,           dC_t = sum_c gy_t h_t.
// A workgroup walks its sequence's tiles from the last to the first.  The
// states come from the forward's kept ones (one per SELECT_CK = one tile), the
// gradient through the later tiles is carried.  Inside a tile the chunks run
// side by side in both directions as in the forward: each wave forms its decays,
// its state from zero and its gradient from zero, one exchange gives both true
// ends, and a second pass forms the states (kept in registers) and then the
// gradients.  dB and dC of the workgroup's channels go to a partial sum.
template <typename Tin, int N, bool VEC>
__global__ __launch_bounds__(512) void k_select_bwd(SelectArgs a) {
  constexpr int CPL = select_block_channels(N) * N / 256, L = 4, W = 8;
  using S = SelTile<N, CPL>;
  constexpr int LN = S::LN, CG = S::CG, CW = S::CW, TL = (L + LN - 1) / LN, TILE = L * W;
  constexpr int VL = CPL / LN > 0 ? CPL / LN : 1;  // channels of a lane after a sum over the states
  static_assert(TILE == SELECT_CK, "a tile starts at a kept state");
  struct WaveLds {
    float dt[L][CW], xu[L][CW], gy[L][CW], yp[L][CW], B[L][N], C[L][N];
  };
  __shared__ __align__(16) WaveLds lds[W];
  __shared__ float4 ex[W][3][CPL][64];  // a chunk's decay product, state and gradient from zero
  __shared__ float4 gb[CPL][64];        // gradient of the state that leaves the tile, decayed

  const int lane = lane_id(), w = wave_id_s(), ng = lane / CG, cg = lane % CG;
  const int Dg = a.D / a.G, nblk = (Dg + CW - 1) / CW, nb = a.G * nblk;
  const int seq = blockIdx.x / nb, blk = blockIdx.x % nb, g = blk / nblk;
  const int cl = g * Dg + (blk % nblk) * CW + cg * CPL;
  const int nv = max(0, min(CPL, (g + 1) * Dg - cl));
  const int cs = nv > 0 ? cl : g * Dg, ns = max(nv, 1);
  int tok0, tok1;
  seq_range(a.cu_seqlens, seq, a.Tseq, a.Ttot, tok0, tok1);
  const int len = tok1 - tok0;
  WaveLds& my = lds[w];

  float A2[CPL][4], dA[CPL][4], bias[CPL], skip[CPL], dD[CPL], db[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = min(cs + i, cs + ns - 1);
    bias[i] = a.bias ? a.bias[c] : 0.f;
    skip[i] = a.Dskip ? a.Dskip[c] : 0.f;
    dD[i] = db[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      A2[i][j] = i < nv ? a.A[(long)c * N + ng * 4 + j] * LOG2E : 0.f;
      dA[i][j] = 0.f;
    }
  }
  if (w == 0) {
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        f[j] = a.dht && i < nv ? a.dht[((long)seq * a.D + cl + i) * N + ng * 4 + j] : 0.f;
      gb[i][lane] = make_float4(f[0], f[1], f[2], f[3]);
    }
  }
  const Tin *u = static_cast<const Tin*>(a.u), *delta = static_cast<const Tin*>(a.delta),
            *z = static_cast<const Tin*>(a.z), *dy = static_cast<const Tin*>(a.dy);
  const Tin *Bm = static_cast<const Tin*>(a.Bm), *Cm = static_cast<const Tin*>(a.Cm);
  const int ntiles = (len + TILE - 1) / TILE;

  Piece<Tin, CPL, VEC> pu[TL], pd[TL], pz[TL], py[TL];
  constexpr int SN = L * N / 64 > 0 ? L * N / 64 : 1;  // states per lane of the chunk's B, C rows
  const int stok = min(lane * SN / N, L - 1), sst = lane * SN % N;
  float pb[SN], pc[SN];
  float4 pk[CPL];  // the kept state at the tile's start
  auto load = [&](int tile) {
    const int t0 = tile * TILE + w * L;
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      const long row = tok0 + min(t0 + min(ng + LN * k, L - 1), len - 1);
      pu[k].load(u + row * a.u_row + cs, ns);
      pd[k].load(delta + row * a.delta_row + cs, ns);
      if (z) pz[k].load(z + row * a.z_row + cs, ns);
      py[k].load(dy + row * a.D + cs, ns);
    }
    const long row = tok0 + min(t0 + stok, len - 1);
#pragma unroll
    for (int e = 0; e < SN; ++e) {
      pb[e] = to_f(Bm[row * a.b_row + g * N + sst + e]);
      pc[e] = to_f(Cm[row * a.c_row + g * N + sst + e]);
    }
    const float* ck = a.ck + ((long)(tok0 / SELECT_CK + seq + tile) * a.D + cs) * N + ng * 4;
#pragma unroll
    for (int i = 0; i < CPL; ++i) pk[i] = *reinterpret_cast<const float4*>(ck + min(i, ns - 1) * N);
  };
  if (ntiles > 0) load(ntiles - 1);
  for (int tile = ntiles - 1; tile >= 0; --tile) {
    const int t0 = tile * TILE + w * L;
    float h[CPL][4], G[CPL][4];
    float4 hk[CPL];
    // per own token: raw u, dt and gy stay in registers; slope = d dt / d raw,
    // and for z: silu(z), silu'(z) dy
    float ou[TL][CPL], oslope[TL][CPL], odz[TL][CPL], odt[TL][CPL], ogy[TL][CPL];
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      const int tl = ng + LN * k;
      const bool ok = tl < L && t0 + tl < len;
      float xu[CPL];
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        const bool on = ok && i < nv;
        const float raw = pd[k].get(i) + bias[i];
        odt[k][i] = on ? (a.softplus ? softplus_acc(raw) : raw) : 0.f;
        oslope[k][i] = a.softplus ? sigmoid_acc(raw) : 1.f;
        ou[k][i] = on ? pu[k].get(i) : 0.f;
        xu[i] = odt[k][i] * ou[k][i];
        float dyv = on ? py[k].get(i) : 0.f;
        odz[k][i] = 0.f;
        if (z) {
          const float zv = on ? pz[k].get(i) : 0.f, sg = sigmoid_acc(zv);
          odz[k][i] = dyv * sg * fmaf(zv, 1.f - sg, 1.f);
          dyv *= zv * sg;
        }
        ogy[k][i] = dyv;
      }
      if (tl < L) {
        lds_put<CPL>(&my.dt[tl][cg * CPL], odt[k]);
        lds_put<CPL>(&my.xu[tl][cg * CPL], xu);
        lds_put<CPL>(&my.gy[tl][cg * CPL], ogy[k]);
      }
    }
    if (lane * SN < L * N) {
      const bool ok = t0 + stok < len;
#pragma unroll
      for (int e = 0; e < SN; ++e) {
        my.B[stok][sst + e] = ok ? pb[e] : 0.f;
        my.C[stok][sst + e] = ok ? pc[e] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < CPL; ++i) hk[i] = pk[i];
    __builtin_amdgcn_wave_barrier();
    if (tile > 0) load(tile - 1);

    // the chunk from zero, forward then backward
    float dec[L][CPL][4], sdt[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      sdt[i] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) h[i][j] = G[i][j] = 0.f;
    }
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
          h[i][j] = fmaf(dec[t][i][j], h[i][j], xu[i] * Bv[j]);
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
        for (int j = 0; j < 4; ++j) G[i][j] = dec[t][i][j] * fmaf(Cv[j], gy[i], G[i][j]);
    }
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      ex[w][0][i][lane] = make_float4(
          __builtin_amdgcn_exp2f(sdt[i] * A2[i][0]), __builtin_amdgcn_exp2f(sdt[i] * A2[i][1]),
          __builtin_amdgcn_exp2f(sdt[i] * A2[i][2]), __builtin_amdgcn_exp2f(sdt[i] * A2[i][3]));
      ex[w][1][i][lane] = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
      ex[w][2][i][lane] = make_float4(G[i][0], G[i][1], G[i][2], G[i][3]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const float4 f = gb[i][lane];
      G[i][0] = f.x;
      G[i][1] = f.y;
      G[i][2] = f.z;
      G[i][3] = f.w;
      h[i][0] = hk[i].x;
      h[i][1] = hk[i].y;
      h[i][2] = hk[i].z;
      h[i][3] = hk[i].w;
    }
    for (int m = 0; m < w; ++m) {
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        const float4 p = ex[m][0][i][lane], f = ex[m][1][i][lane];
        h[i][0] = fmaf(p.x, h[i][0], f.x);
        h[i][1] = fmaf(p.y, h[i][1], f.y);
        h[i][2] = fmaf(p.z, h[i][2], f.z);
        h[i][3] = fmaf(p.w, h[i][3], f.w);
      }
    }
    for (int m = W - 1; m > w; --m) {
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        const float4 p = ex[m][0][i][lane], f = ex[m][2][i][lane];
        G[i][0] = fmaf(p.x, G[i][0], f.x);
        G[i][1] = fmaf(p.y, G[i][1], f.y);
        G[i][2] = fmaf(p.z, G[i][2], f.z);
        G[i][3] = fmaf(p.w, G[i][3], f.w);
      }
    }
    __syncthreads();
    // second pass: the states (hs[t] enters token t)
    float hs[L + 1][CPL][4];
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) hs[0][i][j] = h[i][j];
#pragma unroll
    for (int t = 0; t < L; ++t) {
      __builtin_amdgcn_sched_barrier(0);
      float xu[CPL], Bv[4], Cv[4], s[CPL];
      lds_get<CPL>(&my.xu[t][cg * CPL], xu);
      lds_get<4>(&my.B[t][ng * 4], Bv);
      lds_get<4>(&my.C[t][ng * 4], Cv);
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        s[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          hs[t + 1][i][j] = fmaf(dec[t][i][j], hs[t][i][j], xu[i] * Bv[j]);
          s[i] = fmaf(Cv[j], hs[t + 1][i][j], s[i]);
        }
      }
      if (z) {  // the ungated output, for dz
        spread_sum<CPL, 5, 6 - S::LNB>(s);
        float o[VL];
#pragma unroll
        for (int i = 0; i < VL; ++i) o[i] = s[i];
        const int at = cg * CPL + (LN >= CPL ? ng / (LN / CPL) : ng * VL);
        lds_put<VL>(&my.yp[t][at], o);
      }
    }
    // second pass: the gradients
#pragma unroll
    for (int t = L - 1; t >= 0; --t) {
      __builtin_amdgcn_sched_barrier(0);
      float dt[CPL], xu[CPL], gy[CPL], Bv[4], Cv[4], bc[8], sb[CPL], sa[CPL];
      lds_get<CPL>(&my.dt[t][cg * CPL], dt);
      lds_get<CPL>(&my.xu[t][cg * CPL], xu);
      lds_get<CPL>(&my.gy[t][cg * CPL], gy);
      lds_get<4>(&my.B[t][ng * 4], Bv);
      lds_get<4>(&my.C[t][ng * 4], Cv);
#pragma unroll
      for (int j = 0; j < 8; ++j) bc[j] = 0.f;
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        sb[i] = sa[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float dh = fmaf(Cv[j], gy[i], G[i][j]);
          G[i][j] = dec[t][i][j] * dh;
          const float p = G[i][j] * hs[t][i][j];
          sb[i] = fmaf(dh, Bv[j], sb[i]);
          sa[i] = fmaf(A2[i][j], p, sa[i]);
          dA[i][j] = fmaf(dt[i], p, dA[i][j]);
          bc[j] = fmaf(dh, xu[i], bc[j]);
          bc[4 + j] = fmaf(gy[i], hs[t + 1][i][j], bc[4 + j]);
        }
      }
      // over the states: <B, dh> and <A, p> replace the token's xu and dt
      spread_sum<CPL, 5, 6 - S::LNB>(sb);
      spread_sum<CPL, 5, 6 - S::LNB>(sa);
      float ob[VL], oa[VL];
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        ob[i] = sb[i];
        oa[i] = sa[i];
      }
      const int at = cg * CPL + (LN >= CPL ? ng / (LN / CPL) : ng * VL);
      __builtin_amdgcn_wave_barrier();
      lds_put<VL>(&my.xu[t][at], ob);
      lds_put<VL>(&my.dt[t][at], oa);
      // over the channels: lane cg's top three bits say which of the 8 values it holds
      spread_sum<8, 5 - S::LNB, 0>(bc);
      constexpr int REST = CG / 8;  // lanes with the same value
      if (cg % REST == 0 && t0 + t < len) {
        const int v = cg / REST;
        a.bcp[((long)blk * a.Ttot + tok0 + t0 + t) * (2 * N) + (v >> 2) * N + ng * 4 + (v & 3)] = bc[0];
      }
    }
    if (w == 0) {
#pragma unroll
      for (int i = 0; i < CPL; ++i) gb[i][lane] = make_float4(G[i][0], G[i][1], G[i][2], G[i][3]);
    }
    __builtin_amdgcn_wave_barrier();
    // the own tokens' gradients
#pragma unroll
    for (int k = 0; k < TL; ++k) {
      const int tl = ng + LN * k, t = t0 + tl;
      if (tl < L && t < len) {
        float sb[CPL], sa[CPL], yp[CPL], du[CPL], dd[CPL], dz[CPL];
        lds_get<CPL>(&my.xu[tl][cg * CPL], sb);
        lds_get<CPL>(&my.dt[tl][cg * CPL], sa);
        if (z) lds_get<CPL>(&my.yp[tl][cg * CPL], yp);
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
          du[i] = fmaf(odt[k][i], sb[i], skip[i] * ogy[k][i]);
          dd[i] = fmaf(ou[k][i], sb[i], LN2 * sa[i]) * oslope[k][i];
          dD[i] = fmaf(ogy[k][i], ou[k][i], dD[i]);
          db[i] += dd[i];
          dz[i] = z ? odz[k][i] * fmaf(skip[i], ou[k][i], yp[i]) : 0.f;
        }
        const long at = (long)(tok0 + t) * a.D + cl;
        store_piece<Tin, CPL, VEC>(static_cast<Tin*>(a.du) + at, du, nv);
        store_piece<Tin, CPL, VEC>(static_cast<Tin*>(a.ddelta) + at, dd, nv);
        if (z) store_piece<Tin, CPL, VEC>(static_cast<Tin*>(a.dz) + at, dz, nv);
      }
    }
  }
  // the sequence's parameter gradients: the waves' sums in order, dD and dbias
  // also over the lane groups, which held different tokens
  __syncthreads();
  float4* part = &ex[0][0][0][0];  // [W][CPL][64] dA, then [W][2][CPL][64] floats
  float* pd2 = reinterpret_cast<float*>(part + W * CPL * 64);
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    part[(w * CPL + i) * 64 + lane] = make_float4(dA[i][0], dA[i][1], dA[i][2], dA[i][3]);
    pd2[((w * 2 + 0) * CPL + i) * 64 + lane] = dD[i];
    pd2[((w * 2 + 1) * CPL + i) * 64 + lane] = db[i];
  }
  __syncthreads();
  if (w == 0) {
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      float4 s = part[i * 64 + lane];
      for (int m = 1; m < W; ++m) {
        const float4 v = part[(m * CPL + i) * 64 + lane];
        s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
      }
      if (i < nv) {
        float* p = a.dap + ((long)seq * a.D + cl + i) * (N + 2);
        p[ng * 4] = s.x;
        p[ng * 4 + 1] = s.y;
        p[ng * 4 + 2] = s.z;
        p[ng * 4 + 3] = s.w;
        if (ng == 0) {
          float sd = 0.f, sb = 0.f;
          for (int m = 0; m < W; ++m)
            for (int e = 0; e < LN; ++e) {
              sd += pd2[((m * 2 + 0) * CPL + i) * 64 + e * CG + cg];
              sb += pd2[((m * 2 + 1) * CPL + i) * 64 + e * CG + cg];
            }
          p[N] = sd;
          p[N + 1] = sb;
        }
        if (a.dh0) {
          const float4 f = gb[i][lane];
          float* q = a.dh0 + ((long)seq * a.D + cl + i) * N + ng * 4;
          q[0] = f.x;
          q[1] = f.y;
          q[2] = f.z;
          q[3] = f.w;
        }
      }
    }
  }
}

// dB, dC of every (token, group, state): the channel blocks' partial sums in order.
template <typename Tin>
__global__ __launch_bounds__(256) void k_select_dbc(SelectArgs a) {
  const int N2 = 2 * a.N;
  const long n = (long)a.Ttot * a.G * N2;
  const long e = (long)blockIdx.x * 256 + threadIdx.x;
  if (e >= n) return;
  const int s = e % N2;
  const long tg = e / N2;
  const int g = tg / a.Ttot;
  const long t = tg % a.Ttot;
  const float* p = a.bcp + ((long)g * a.nblk * a.Ttot + t) * N2 + s;
  float sum = 0.f;
  for (int b = 0; b < a.nblk; ++b) sum += p[(long)b * a.Ttot * N2];
  Tin* out = static_cast<Tin*>(s < a.N ? a.dB : a.dC);
  store_elem(out + (t * a.G + g) * a.N + (s < a.N ? s : s - a.N), sum);
}

// dA, dD and dbias: the sequences' partial sums in order.
__global__ __launch_bounds__(256) void k_select_dparam(SelectArgs a) {
  const int N2 = a.N + 2;
  const long n = (long)a.D * N2;
  const long e = (long)blockIdx.x * 256 + threadIdx.x;
  if (e >= n) return;
  float sum = 0.f;
  for (int s = 0; s < a.S; ++s) sum += a.dap[s * n + e];
  const int k = e % N2;
  const long c = e / N2;
  if (k < a.N) a.dA[c * a.N + k] = sum;
  else if (k == a.N) { if (a.dD) a.dD[c] = sum; }
  else if (a.dbias) a.dbias[c] = sum;
}

// One token per row: a lane holds 4 states of one channel, consecutive lanes
// consecutive states, so that a wave reads and writes whole kilobytes of the state.
template <typename Tin, int N>
__global__ __launch_bounds__(256) void k_select_step(SelectArgs a) {
  constexpr int LN = N / 4;
  const int nbx = (a.D * LN + 255) / 256;  // workgroups per row
  const int row = blockIdx.x / nbx, e = (blockIdx.x - row * nbx) * 256 + threadIdx.x;
  const int c = e / LN, ng = e % LN;
  const bool on = c < a.D;  // whole lane groups: a channel's lanes agree
  const int slot = a.slots ? a.slots[row] : row;
  Tin* y = static_cast<Tin*>(a.y) + (long)row * a.D + c;
  if (slot < 0 || slot >= a.num_slots) {  // padding
    if (on && ng == 0) store_elem(y, 0.f);
    return;
  }
  const int cc = on ? c : a.D - 1, g = cc / (a.D / a.G);
  const float uv = to_f(static_cast<const Tin*>(a.u)[row * a.u_row + cc]);
  float raw = to_f(static_cast<const Tin*>(a.delta)[row * a.delta_row + cc]);
  if (a.bias) raw += a.bias[cc];
  const float dt = a.softplus ? softplus_acc(raw) : raw, xu = dt * uv;
  const Tin* Bp = static_cast<const Tin*>(a.Bm) + row * a.b_row + g * N + ng * 4;
  const Tin* Cp = static_cast<const Tin*>(a.Cm) + row * a.c_row + g * N + ng * 4;
  const float* Ap = a.A + (long)cc * N + ng * 4;
  float* hp = a.state + ((long)slot * a.D + cc) * N + ng * 4;
  float h[4], s = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    h[j] = fmaf(__builtin_amdgcn_exp2f(dt * (Ap[j] * LOG2E)), hp[j], xu * to_f(Bp[j]));
    s = fmaf(to_f(Cp[j]), h[j], s);
  }
  if (on) {
#pragma unroll
    for (int j = 0; j < 4; ++j) hp[j] = h[j];
  }
  s = xsum<0>(s);
  if constexpr (LN >= 4) s = xsum<1>(s);
  if constexpr (LN >= 8) s = xsum<2>(s);
  if (on && ng == 0) {
    float v = a.Dskip ? fmaf(a.Dskip[cc], uv, s) : s;
    if (a.z) {
      const float zv = to_f(static_cast<const Tin*>(a.z)[row * a.z_row + cc]);
      v *= zv * sigmoid_acc(zv);
    }
    store_elem(y, v);
  }
}

// Whether every row piece of C channels may be loaded at once.
static bool rows_vec(const SelectArgs& a, int C, bool bwd) {
  const long eb = a.bf16 ? 2 : 4, m = C * eb;
  auto ok = [&](const void* p, long row) { return !p || ((uintptr_t)p % m == 0 && row % C == 0); };
  bool v = (a.D / a.G) % C == 0 && ok(a.u, a.u_row) && ok(a.delta, a.delta_row) && ok(a.z, a.z_row);
  if (!bwd) return v && ok(a.y, a.D);
  return v && ok(a.dy, a.D) && ok(a.du, a.D) && ok(a.ddelta, a.D) && ok(a.dz, a.D);
}

template <typename Tin, int N>
static hipError_t run_fwd(const SelectArgs& a) {
  constexpr int CPL = 4, L = 8, W = 8, CW = SelTile<N, CPL>::CW;
  const int Dg = a.D / a.G;
  const long grid = (long)a.S * a.G * ((Dg + CW - 1) / CW);
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (rows_vec(a, CPL, false))
    k_select_fwd<Tin, N, CPL, L, W, true><<<(unsigned)grid, 64 * W, 0, a.stream>>>(a);
  else
    k_select_fwd<Tin, N, CPL, L, W, false><<<(unsigned)grid, 64 * W, 0, a.stream>>>(a);
  return hipGetLastError();
}

template <typename Tin, int N>
static hipError_t run_bwd(const SelectArgs& a) {
  const long grid = (long)a.S * a.G * a.nblk;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (grid > 0) {
    if (rows_vec(a, select_block_channels(N) * N / 256, true)) k_select_bwd<Tin, N, true><<<(unsigned)grid, 512, 0, a.stream>>>(a);
    else k_select_bwd<Tin, N, false><<<(unsigned)grid, 512, 0, a.stream>>>(a);
  }
  const long nbc = (long)a.Ttot * a.G * 2 * N, np = (long)a.D * (N + 2);
  if (nbc > 0) k_select_dbc<Tin><<<(unsigned)((nbc + 255) / 256), 256, 0, a.stream>>>(a);
  k_select_dparam<<<(unsigned)((np + 255) / 256), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

template <typename Tin, int N>
static hipError_t run_step(const SelectArgs& a) {
  const long grid = ((long)a.D * (N / 4) + 255) / 256 * a.S;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  k_select_step<Tin, N><<<(unsigned)grid, 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

#define SELECT_DISPATCH(fn, a)                                                              \
  ((a).N == 8    ? ((a).bf16 ? fn<bf16_t, 8>(a) : fn<float, 8>(a))                          \
   : (a).N == 16 ? ((a).bf16 ? fn<bf16_t, 16>(a) : fn<float, 16>(a))                        \
   : (a).N == 32 ? ((a).bf16 ? fn<bf16_t, 32>(a) : fn<float, 32>(a)) : hipErrorInvalidValue)

hipError_t launch_select_fwd(const SelectArgs& a) {
  return a.S == 0 ? hipSuccess : SELECT_DISPATCH(run_fwd, a);
}
hipError_t launch_select_bwd(const SelectArgs& a) { return SELECT_DISPATCH(run_bwd, a); }
hipError_t launch_select_step(const SelectArgs& a) {
  return a.S == 0 ? hipSuccess : SELECT_DISPATCH(run_step, a);
}

}  // namespace comba
