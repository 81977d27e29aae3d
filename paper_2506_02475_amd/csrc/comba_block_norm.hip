// The norms after and before a block, fused with the gate, the residual scale and the
// residual stream.  Per token, over its C channels:
//
//   p = y rstd(y) w1,   t = p act(z),   r = x + s t,   n = r rstd(r) w2
//   dr' = dr + rstd(r) (dn w2 - rh mean(dn w2 rh)),  rh = r rstd(r);   dx = dr'
//   dt = dr' s,  dz = dt p act'(z),  dp = dt act(z),
//   dy = rstd(y) (dp w1 - yh mean(dp w1 yh)),        yh = y rstd(y)
//   dw2 = sum dn rh,  ds = sum dr' t,  dw1 = sum dp yh      (over the tokens)
//
// Bound by bytes: every value is read and written once.  A row lies in the registers
// of a team (16 lanes, a wave, or a workgroup); a team walks rows with the next row's loads
// in flight, and keeps the parameters and (backward) their gradients' sums in registers.
// Gated, both norms, bf16: 16,384 rows of 4,096 channels forward 124 us (5.4 TB/s), backward
// 247 and 5 for the sums (4.3 TB/s); of 2,048 with an fp32 stream forward 92 (5.1 TB/s).
#include "comba_block_launch.h"
#include "comba_layer_device.hpp"

namespace comba {

constexpr int BN_C = 4;        // channels of an aligned piece
constexpr int BN_WIDE = 1024;  // threads where a row does not fit registers

// Sums of V values over the team, the same in every thread.  `turn` alternates between
// two places in LDS, so that one barrier a sum suffices: a place is written again only
// behind the other's barrier, which every thread reaches after reading the first.
template <int TEAM, int V>
__device__ __forceinline__ void bn_sum(float (&x)[V], float (*lds)[2][16], int& turn) {
#pragma unroll
  for (int v = 0; v < V; ++v) x[v] = team_sum(x[v], TEAM < 64 ? TEAM : 64);
  if constexpr (TEAM > 64) {
    if (lane_id() == 0) {
#pragma unroll
      for (int v = 0; v < V; ++v) lds[turn][v][wave_id()] = x[v];
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < TEAM / 64; ++i) s += lds[turn][v][i];
      x[v] = s;
    }
    turn ^= 1;
  }
}

template <typename Tx, typename Ty, int KV, int C, int TEAM, bool BWD>
__global__ __launch_bounds__(TEAM > 64 ? TEAM : 256) void k_block_norm(BlockNormArgs a, int chunks) {
  __shared__ float lds[2][2][16];
  int turn = 0;
  const int chunk = TEAM > 64 ? blockIdx.x : blockIdx.x * (256 / TEAM) + threadIdx.x / TEAM;
  const int l = threadIdx.x & (TEAM - 1);
  if (chunk >= chunks) return;  // whole teams
  const Tx *xt = static_cast<const Tx*>(a.x), *drt = static_cast<const Tx*>(a.dr);
  const Ty *yt = static_cast<const Ty*>(a.y), *zt = static_cast<const Ty*>(a.z), *dnt = static_cast<const Ty*>(a.dn);
  // (backward: a norm of which nothing comes back takes no part)
  const bool post = a.w1 != nullptr, pre = BWD ? a.dn != nullptr : a.w2 != nullptr;
  int c[KV], nv[KV];
  float w1[KV][C], sc[KV][C], w2[KV][C], d1[KV][C], ds[KV][C], d2[KV][C];
#pragma unroll
  for (int k = 0; k < KV; ++k) {
    const int at = (k * TEAM + l) * C;
    nv[k] = at < a.C ? C : 0;
    c[k] = nv[k] > 0 ? at : 0;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const bool on = nv[k] > 0;
      w1[k][i] = on ? (post ? a.w1[c[k] + i] : 1.f) : 0.f;
      sc[k][i] = on ? (a.sc ? a.sc[c[k] + i] : 1.f) : 0.f;
      w2[k][i] = on && pre ? a.w2[c[k] + i] : 0.f;
      d1[k][i] = ds[k][i] = d2[k][i] = 0.f;
    }
  }
  const float inv = 1.f / a.C;
  Piece<Ty, C, true> py[KV], pz[KV], pn[KV];
  Piece<Tx, C, true> px[KV], pr[KV];
  auto load = [&](long r) {
#pragma unroll
    for (int k = 0; k < KV; ++k) {
      py[k].load(yt + r * a.y_row + c[k], C);
      if (zt) pz[k].load(zt + r * a.z_row + c[k], C);
      if (xt) px[k].load(xt + r * a.x_row + c[k], C);
      if constexpr (BWD) {
        if (drt) pr[k].load(drt + r * a.C + c[k], C);
        if (dnt) pn[k].load(dnt + r * a.C + c[k], C);
      }
    }
  };
  load(chunk);
  for (long r = chunk; r < a.rows; r += chunks) {
    float y[KV][C], z[KV][C], x[KV][C], dr[KV][C], dn[KV][C], sum[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KV; ++k)
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const bool on = nv[k] > 0;
        y[k][i] = on ? py[k].get(i) : 0.f;
        z[k][i] = on && zt ? pz[k].get(i) : 0.f;
        x[k][i] = on && xt ? px[k].get(i) : 0.f;
        if constexpr (BWD) {
          dr[k][i] = on && drt ? pr[k].get(i) : 0.f;
          dn[k][i] = on && dnt ? pn[k].get(i) : 0.f;
        }
        sum[0] = fmaf(y[k][i], y[k][i], sum[0]);
      }
    if (r + chunks < a.rows) load(r + chunks);
    float r1 = 1.f;
    if (post) {
      float s[1] = {sum[0]};
      bn_sum<TEAM>(s, lds, turn);
      r1 = rsqrtf(s[0] * inv + a.eps);
    }
    // y becomes yh, x the new stream
    sum[0] = 0.f;
#pragma unroll
    for (int k = 0; k < KV; ++k)
#pragma unroll
      for (int i = 0; i < C; ++i) {
        y[k][i] *= r1;
        const float p = y[k][i] * w1[k][i];
        const float t = zt ? p * act_of(a.act, z[k][i]) : p;
        x[k][i] = fmaf(t, sc[k][i], x[k][i]);
        sum[0] = fmaf(x[k][i], x[k][i], sum[0]);
        if constexpr (BWD) sum[1] = fmaf(dn[k][i] * w2[k][i], x[k][i], sum[1]);
      }
    if constexpr (!BWD) {
#pragma unroll
      for (int k = 0; k < KV; ++k) store_piece<Tx, C, true>(static_cast<Tx*>(a.r) + r * a.C + c[k], x[k], nv[k]);
    }
    if (!BWD && !pre) continue;
    float r2 = 0.f, m2 = 0.f;
    if (pre) {
      bn_sum<TEAM>(sum, lds, turn);
      r2 = rsqrtf(sum[0] * inv + a.eps);
      m2 = sum[1] * r2 * inv;
    } else {  // (Inf times the r2 of zero would be NaN)
#pragma unroll
      for (int k = 0; k < KV; ++k)
#pragma unroll
        for (int i = 0; i < C; ++i) x[k][i] = 0.f;
    }
    if constexpr (!BWD) {
#pragma unroll
      for (int k = 0; k < KV; ++k) {
        float n[C];
#pragma unroll
        for (int i = 0; i < C; ++i) n[i] = x[k][i] * r2 * w2[k][i];
        store_piece<Ty, C, true>(static_cast<Ty*>(a.n) + r * a.C + c[k], n, nv[k]);
      }
    } else {
      float s1[1] = {0.f};
#pragma unroll
      for (int k = 0; k < KV; ++k) {
        float dz[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const float rh = x[k][i] * r2;
          d2[k][i] = fmaf(dn[k][i], rh, d2[k][i]);
          dr[k][i] += r2 * (dn[k][i] * w2[k][i] - rh * m2);
          const float p = y[k][i] * w1[k][i], dt = dr[k][i] * sc[k][i];
          float gate = 1.f, slope = 0.f;
          if (zt) slope = act_slope(a.act, z[k][i], gate);
          ds[k][i] = fmaf(dr[k][i], p * gate, ds[k][i]);
          dz[i] = dt * p * slope;
          const float dp = dt * gate;
          d1[k][i] = fmaf(dp, y[k][i], d1[k][i]);
          dn[k][i] = dp * w1[k][i];
          s1[0] = fmaf(dn[k][i], y[k][i], s1[0]);
        }
        if (zt) store_piece<Ty, C, true>(static_cast<Ty*>(a.dz) + r * a.C + c[k], dz, nv[k]);
        if (a.dx) store_piece<Tx, C, true>(static_cast<Tx*>(a.dx) + r * a.C + c[k], dr[k], nv[k]);
      }
      float m1 = 0.f;
      if (post) {
        bn_sum<TEAM>(s1, lds, turn);
        m1 = s1[0] * inv;
      } else {  // (an Inf in y times the m1 of zero would be NaN)
#pragma unroll
        for (int k = 0; k < KV; ++k)
#pragma unroll
          for (int i = 0; i < C; ++i) y[k][i] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < KV; ++k) {
        float dy[C];
#pragma unroll
        for (int i = 0; i < C; ++i) dy[i] = r1 * (dn[k][i] - y[k][i] * m1);
        store_piece<Ty, C, true>(static_cast<Ty*>(a.dy) + r * a.C + c[k], dy, nv[k]);
      }
    }
  }
  if constexpr (BWD) {
    float* part = a.part + (long)chunk * 3 * a.C;
#pragma unroll
    for (int k = 0; k < KV; ++k)
#pragma unroll
      for (int i = 0; i < C; ++i)
        if (nv[k] > 0) {
          if (a.dw1) part[c[k] + i] = d1[k][i];
          if (a.dsc) part[a.C + c[k] + i] = ds[k][i];
          if (a.dw2) part[2 * a.C + c[k] + i] = d2[k][i];
        }
  }
}

// Rows whose values in fp32 do not fit registers: a workgroup a row, which forms them again
// for every sum from what it loaded: KV pieces a thread, as they are, with the parameters'
// gradients in registers (8,192 rows of 8,192 channels, forward and backward, 444 us; with
// everything in fp32 it spilled, 861; with parameters loaded value by value 1,083); KV 0:
// from the caches, those gradients in its partial row.
template <typename Tx, typename Ty, int KV, int C, bool BWD>
__global__ __launch_bounds__(BN_WIDE) void k_block_norm_wide(BlockNormArgs a, int chunks) {
  __shared__ float lds[2][2][16];
  int turn = 0;
  constexpr int N = KV > 0 ? KV : 1;
  const int chunk = blockIdx.x;
  const Tx *xt = static_cast<const Tx*>(a.x), *drt = static_cast<const Tx*>(a.dr);
  const Ty *yt = static_cast<const Ty*>(a.y), *zt = static_cast<const Ty*>(a.z), *dnt = static_cast<const Ty*>(a.dn);
  // (backward: a norm of which nothing comes back takes no part)
  const bool post = a.w1 != nullptr, pre = BWD ? a.dn != nullptr : a.w2 != nullptr;
  const float inv = 1.f / a.C;
  float* part = BWD ? a.part + (long)chunk * 3 * a.C : nullptr;
  Piece<Ty, C, true> py[N], pz[N], pn[N];
  Piece<Tx, C, true> px[N], pr[N];
  float d1[N][C], ds[N][C], d2[N][C];
  // fn(number, first channel) for every piece of the thread
  auto pieces = [&](auto fn) {
    if constexpr (KV > 0) {
#pragma unroll
      for (int k = 0; k < KV; ++k) {
        const int c = (k * BN_WIDE + (int)threadIdx.x) * C;
        if (c < a.C) fn(k, c);
      }
    } else {
      for (int c = threadIdx.x * C; c < a.C; c += BN_WIDE * C) fn(0, c);
    }
  };
  auto load_y = [&](long r, int k, int c) { py[k].load(yt + r * a.y_row + c, C); };
  auto load_rest = [&](long r, int k, int c) {
    if (zt) pz[k].load(zt + r * a.z_row + c, C);
    if (xt) px[k].load(xt + r * a.x_row + c, C);
    if constexpr (BWD) {
      if (dnt) pn[k].load(dnt + r * a.C + c, C);
      else pn[k].zero();
      if (drt) pr[k].load(drt + r * a.C + c, C);
    }
  };
  if constexpr (BWD) {
    pieces([&](int k, int c) {
#pragma unroll
      for (int i = 0; i < C; ++i) {
        if constexpr (KV > 0) d1[k][i] = ds[k][i] = d2[k][i] = 0.f;
        else part[c + i] = part[a.C + c + i] = part[2 * a.C + c + i] = 0.f;
      }
    });
  }
  for (long r = chunk; r < a.rows; r += chunks) {
    float r1 = 1.f, r2 = 0.f, m1 = 0.f, m2 = 0.f;
    if constexpr (KV > 0) {
      pieces([&](int k, int c) {
        load_y(r, k, c);
        load_rest(r, k, c);
      });
    }
    if (post) {
      float s[1] = {0.f};
      pieces([&](int k, int c) {
        if constexpr (KV == 0) load_y(r, k, c);
#pragma unroll
        for (int i = 0; i < C; ++i) s[0] = fmaf(py[k].get(i), py[k].get(i), s[0]);
      });
      bn_sum<BN_WIDE>(s, lds, turn);
      r1 = rsqrtf(s[0] * inv + a.eps);
    }
    // fn(i, channel, yh, gate, its slope, stream) for every channel of a piece, its
    // parameters in w1, sc and w2
    Piece<float, C, true> w1, sc, w2;
    auto stream = [&](int k, int c, auto fn) {
      if constexpr (KV == 0) {
        load_y(r, k, c);
        load_rest(r, k, c);
      }
      if (post) w1.load(a.w1 + c, C);
      if (a.sc) sc.load(a.sc + c, C);
      if (pre) w2.load(a.w2 + c, C);
      else w2.zero();
#pragma unroll
      for (int i = 0; i < C; ++i) {
        if (!post) w1.r[i] = __float_as_uint(1.f);
        if (!a.sc) sc.r[i] = __float_as_uint(1.f);
      }
#pragma unroll
      for (int i = 0; i < C; ++i) {
        float gate = 1.f, slope = 0.f;
        if (zt) slope = act_slope(a.act, pz[k].get(i), gate);
        const float yh = py[k].get(i) * r1, t = yh * w1.get(i) * gate;
        fn(i, c + i, yh, gate, slope, fmaf(t, sc.get(i), xt ? px[k].get(i) : 0.f));
      }
    };
    float s2[2] = {0.f, 0.f};
    pieces([&](int k, int c) {
      float out[C];
      stream(k, c, [&](int i, int, float, float, float, float v) {
        out[i] = v;
        s2[0] = fmaf(v, v, s2[0]);
        if constexpr (BWD) s2[1] = fmaf(pn[k].get(i) * w2.get(i), v, s2[1]);
      });
      if constexpr (!BWD) store_piece<Tx, C, true>(static_cast<Tx*>(a.r) + r * a.C + c, out, C);
    });
    if (pre) {
      bn_sum<BN_WIDE>(s2, lds, turn);
      r2 = rsqrtf(s2[0] * inv + a.eps);
      m2 = s2[1] * r2 * inv;
    }
    if constexpr (!BWD) {
      if (!pre) continue;
      pieces([&](int k, int c) {
        float n[C];
        stream(k, c, [&](int i, int, float, float, float, float v) { n[i] = v * r2 * w2.get(i); });
        store_piece<Ty, C, true>(static_cast<Ty*>(a.n) + r * a.C + c, n, C);
      });
    } else {
      // fn(i, channel, yh, dn rh, dr', t, dz, dp) for every channel of a piece
      auto grad = [&](int k, int c, auto fn) {
        stream(k, c, [&](int i, int at, float yh, float gate, float slope, float v) {
          float dr = drt ? pr[k].get(i) : 0.f, dw2 = 0.f;
          if (pre) {  // (as zeros the terms would be NaN where a row holds an Inf)
            const float rh = v * r2, dn = pn[k].get(i);
            dr += r2 * (dn * w2.get(i) - rh * m2);
            dw2 = dn * rh;
          }
          const float p = yh * w1.get(i), dt = dr * sc.get(i);
          fn(i, at, yh, dw2, dr, p * gate, dt * p * slope, dt * gate);
        });
      };
      float s1[1] = {0.f};
      pieces([&](int k, int c) {
        float dx[C], dz[C];
        grad(k, c, [&](int i, int at, float yh, float dw2, float dr, float t, float d, float dp) {
          dx[i] = dr;
          dz[i] = d;
          s1[0] = fmaf(dp * w1.get(i), yh, s1[0]);
          float &g1 = KV > 0 ? d1[k][i] : part[at], &gs = KV > 0 ? ds[k][i] : part[a.C + at],
                &g2 = KV > 0 ? d2[k][i] : part[2 * a.C + at];
          g1 = fmaf(dp, yh, g1);
          gs = fmaf(dr, t, gs);
          g2 += dw2;
        });
        if (zt) store_piece<Ty, C, true>(static_cast<Ty*>(a.dz) + r * a.C + c, dz, C);
        if (a.dx) store_piece<Tx, C, true>(static_cast<Tx*>(a.dx) + r * a.C + c, dx, C);
      });
      if (post) {
        bn_sum<BN_WIDE>(s1, lds, turn);
        m1 = s1[0] * inv;
      }
      pieces([&](int k, int c) {
        float dy[C];
        grad(k, c, [&](int i, int, float yh, float, float, float, float, float dp) {
          dy[i] = pre || post ? r1 * (dp * w1.get(i) - yh * m1) : dp;  // (likewise)
        });
        store_piece<Ty, C, true>(static_cast<Ty*>(a.dy) + r * a.C + c, dy, C);
      });
    }
  }
  if constexpr (BWD && KV > 0) {
    pieces([&](int k, int c) {
#pragma unroll
      for (int i = 0; i < C; ++i) {
        part[c + i] = d1[k][i];
        part[a.C + c + i] = ds[k][i];
        part[2 * a.C + c + i] = d2[k][i];
      }
    });
  }
}

// The parameters' gradients: the chunks' partial sums, each of 16 waves every 16th in
// order, then the waves in order.
constexpr int BN_WAVES = 16;
__global__ __launch_bounds__(64 * BN_WAVES) void k_block_norm_dw(BlockNormArgs a) {
  __shared__ float part[BN_WAVES][64];
  const int lane = lane_id(), w = wave_id_s(), which = blockIdx.y, e = blockIdx.x * 64 + lane;
  float* out = which == 0 ? a.dw1 : which == 1 ? a.dsc : a.dw2;
  if (!out) return;  // the whole workgroup
  float s = 0.f;
  if (e < a.C) {
#pragma unroll 8
    for (int r = w; r < a.blocks; r += BN_WAVES) s += a.part[((long)r * 3 + which) * a.C + e];
  }
  part[w][lane] = s;
  __syncthreads();
  if (w == 0 && e < a.C) {
    for (int i = 1; i < BN_WAVES; ++i) s += part[i][lane];
    out[e] = s;
  }
}

// The team of a row, and how many teams walk the rows: 1,024 lanes per CU, or 512 where a
// lane has two pieces, whose loads in flight are enough at that (bf16, gated, both norms,
// 512 / 1,024 / 2,048 lanes: 65,536 rows of 512 channels forward 64 / 69 / 66 us, forward and
// backward 186 / 206 / 230; 16,384 of 2,048 65 / 71 / 69 and 183 / 191 / 204; one piece, 32,768
// of 1,024 73 / 64 / 68 and 205 / 183 / 199).
struct BnTeam {
  int team, kv, chunks;
};
static BnTeam bn_team(const BlockNormArgs& a) {
  BnTeam t;
  const int pieces = (a.C + BN_C - 1) / BN_C;
  t.team = pieces <= 32 ? 16 : pieces <= 128 ? 64 : pieces <= 512 ? 256 : pieces <= 1024 ? 512 : 1024;
  t.kv = pieces <= t.team ? 1 : pieces <= 2 * t.team ? 2 : 0;
  const long lanes = t.kv == 2 && t.team < 1024 ? 512 : 1024, chunks = 256L * lanes / t.team;
  t.chunks = (int)(chunks > a.rows ? a.rows : chunks);
  return t;
}
int block_norm_bwd_blocks(const BlockNormArgs& a) { return a.rows > 0 ? bn_team(a).chunks : 0; }

template <typename Tx, typename Ty, bool BWD>
static hipError_t run_block_norm(const BlockNormArgs& a0) {
  BlockNormArgs a = a0;
  if (a.rows > 0) {
    const BnTeam t = bn_team(a);
    a.blocks = t.chunks;
    auto ok = [&](const void* p, size_t eb, long row) {
      return !p || ((uintptr_t)p % (BN_C * eb) == 0 && row % BN_C == 0);
    };
    const bool vec = a.C % BN_C == 0 && ok(a.y, sizeof(Ty), a.y_row) && ok(a.z, sizeof(Ty), a.z_row) &&
                     ok(a.x, sizeof(Tx), a.x_row) && ok(a.r, sizeof(Tx), 0) && ok(a.n, sizeof(Ty), 0) &&
                     ok(a.dr, sizeof(Tx), 0) && ok(a.dn, sizeof(Ty), 0) && ok(a.dy, sizeof(Ty), 0) &&
                     ok(a.dx, sizeof(Tx), 0) && ok(a.dz, sizeof(Ty), 0) && ok(a.w1, 4, 0) && ok(a.sc, 4, 0) &&
                     ok(a.w2, 4, 0);
    const int each = t.team > 64 ? 1 : 256 / t.team;  // teams of a workgroup
    const unsigned grid = (t.chunks + each - 1) / each;
#define BN_LAUNCH(KV, TEAM)                                                                              \
  if (vec) k_block_norm<Tx, Ty, KV, BN_C, TEAM, BWD><<<grid, TEAM > 64 ? TEAM : 256, 0, a.stream>>>(a, t.chunks); \
  else k_block_norm<Tx, Ty, KV * BN_C, 1, TEAM, BWD><<<grid, TEAM > 64 ? TEAM : 256, 0, a.stream>>>(a, t.chunks);
    if (t.team == 16 && t.kv == 1) { BN_LAUNCH(1, 16) }
    else if (t.team == 16) { BN_LAUNCH(2, 16) }
    else if (t.team == 64 && t.kv == 1) { BN_LAUNCH(1, 64) }
    else if (t.team == 64) { BN_LAUNCH(2, 64) }
    else if (t.team == 256 && t.kv == 1) { BN_LAUNCH(1, 256) }
    else if (t.team == 256) { BN_LAUNCH(2, 256) }
    else if (t.team == 512) { BN_LAUNCH(2, 512) }
#undef BN_LAUNCH
    else if (t.kv && !BWD && vec) k_block_norm<Tx, Ty, 2, BN_C, 1024, false><<<grid, 1024, 0, a.stream>>>(a, t.chunks);
#define BN_LAUNCH(KV, C) k_block_norm_wide<Tx, Ty, KV, C, BWD><<<grid, BN_WIDE, 0, a.stream>>>(a, t.chunks)
    else if (t.kv && vec) BN_LAUNCH(2, BN_C);
    else if (t.kv) BN_LAUNCH(8, 1);
    else if (vec) BN_LAUNCH(0, BN_C);
    else BN_LAUNCH(0, 1);
#undef BN_LAUNCH
  }
  if (BWD && (a.dw1 || a.dsc || a.dw2))
    k_block_norm_dw<<<dim3((unsigned)((a.C + 63) / 64), 3), 64 * BN_WAVES, 0, a.stream>>>(a);
  return hipGetLastError();
}

#define BN_DISPATCH(BWD, a)                              \
  ((a).x_bf16 ? run_block_norm<bf16_t, bf16_t, BWD>(a)   \
   : (a).bf16 ? run_block_norm<float, bf16_t, BWD>(a) : run_block_norm<float, float, BWD>(a))

hipError_t launch_block_norm_fwd(const BlockNormArgs& a) { return BN_DISPATCH(false, a); }
hipError_t launch_block_norm_bwd(const BlockNormArgs& a) { return BN_DISPATCH(true, a); }

}  // namespace comba
