// Group norm per token, channels last: mean and variance over the m = C / G
// channels of a group of one token, then weight and bias, then an activation of
// the result, or a gate y = n act(z):
//
//   n = (x - mean) rstd w + b,   y = act(n)  |  n act(z).
//
// Bound by bytes: every value is read and written once.  A group's channels lie
// in the registers of a team of 1..64 lanes (a power of two) or of a workgroup of
// 256 or 512, KV pieces of C channels per lane, so that mean and variance are two passes
// over registers.  A team keeps its group and walks rows, the next row's loads in
// flight, with weight and bias (backward: and their gradients' sums) in registers.
// 16,384 x 4,096 channels in groups of 128, gated, bf16: forward 84 us (4.8 TB/s),
// backward 134 us and 5 for the sums (5.0 TB/s); x in fp32, 2,048 channels: 45 us.
//
// Groups of more than 8,192 channels read x again from the caches
// (k_group_norm_wide), at a higher cost: 8,192 rows of one group of 8,192 channels
// take 87 us forward and 170 backward in registers, of 12,000 from the caches 336
// and 966, 2.8 and 4.9 times their bytes at the copy rate (dw and db are read and
// written per row there, and the gradient is formed twice); one group of 4,096 from the
// caches 443 and 929 for 16,384 rows, not 88 and 158.  An odd width takes one channel a
// piece: 8,192 rows of 8,191 channels 136 and 218 in bf16 (whose backward keeps 12 of its
// registers in scratch), 152 and 290 in fp32.
#include "comba_layer_device.hpp"
#include "comba_layer_launch.h"

namespace comba {

constexpr int GN_C = 4;        // channels of an aligned piece
constexpr int GN_WIDE = 1024;  // threads where a group's channels do not fit registers

// Sum over the lanes of a team (team: a power of two up to 64), the same in every lane.
__device__ __forceinline__ float team_sum(float x, int team) {
  if (team > 1) x = xsum<0>(x);
  if (team > 2) x = xsum<1>(x);
  if (team > 4) x = xsum<2>(x);
  if (team > 8) x = xsum<3>(x);
  if (team > 16) x = xsum<4>(x);
  if (team > 32) x = xsum<5>(x);
  return x;
}

// act(t) and, for the backward, its slope.
__device__ __forceinline__ float act_of(comba_activation act, float t) {
  if (act == COMBA_ACT_NONE) return t;
  const float s = sigmoid_acc(t);
  return act == COMBA_ACT_SILU ? t * s : s;
}
__device__ __forceinline__ float act_slope(comba_activation act, float t, float& y) {
  if (act == COMBA_ACT_NONE) {
    y = t;
    return 1.f;
  }
  const float s = sigmoid_acc(t);
  if (act == COMBA_ACT_SILU) {
    y = t * s;
    return s * fmaf(t, 1.f - s, 1.f);
  }
  y = s;
  return s * (1.f - s);
}

// Sum over a workgroup of TH threads, the same in every thread.
template <int TH>
__device__ __forceinline__ float block_sum(float x, float* lds) {
  x = team_sum(x, 64);
  if (lane_id() == 0) lds[wave_id()] = x;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < TH / 64; ++i) s += lds[i];
  __syncthreads();
  return s;
}

// The same over the team: a wave's lanes (TEAM 0), or a workgroup of TEAM threads.
template <int TEAM>
__device__ __forceinline__ float gn_sum(float x, int team, float* lds) {
  if constexpr (TEAM > 0) return block_sum<TEAM>(x, lds);
  return team_sum(x, team);
}

struct GnTeam {
  int team;    // lanes
  int chunks;  // row chunks: team (group, chunk) takes rows chunk, chunk + chunks, ..
};

template <typename Tx, typename To, int KV, int C, int TEAM, bool BWD>
__global__ __launch_bounds__(TEAM > 0 ? TEAM : 256) void k_group_norm(GroupNormArgs a, GnTeam tm) {
  __shared__ float lds[TEAM / 64 + 1];
  const int m = a.C / a.G, team = TEAM > 0 ? TEAM : tm.team;
  const long id = ((long)blockIdx.x * (TEAM > 0 ? TEAM : 256) + threadIdx.x) / team;
  const int l = threadIdx.x & (team - 1);
  const int g = id % a.G, chunk = id / a.G;
  if (chunk >= tm.chunks) return;  // whole teams
  // where not everything fits registers: each row loaded when it is due, and the
  // sums of dw and db in LDS
  constexpr bool LEAN = BWD && TEAM == 512 && C == 1;
  __shared__ float kept[2][LEAN ? KV : 1][LEAN ? TEAM : 1];
  int c[KV], nv[KV];
  float w[KV][C], b[KV][C], dw[KV][C], db[KV][C];
#pragma unroll
  for (int k = 0; k < KV; ++k) {
    const int at = (k * team + l) * C;  // in the group
    nv[k] = at < m ? C : 0;
    c[k] = g * m + (nv[k] > 0 ? at : 0);
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const bool on = nv[k] > 0;
      w[k][i] = on ? (a.w ? a.w[c[k] + i] : 1.f) : 0.f;
      b[k][i] = on && a.b ? a.b[c[k] + i] : 0.f;
      if constexpr (LEAN) kept[0][k][l] = kept[1][k][l] = 0.f;
      else dw[k][i] = db[k][i] = 0.f;
    }
  }
  const float inv = 1.f / m;
  const Tx* x = static_cast<const Tx*>(a.x);
  const To *z = static_cast<const To*>(a.z), *dy = static_cast<const To*>(a.dy);
  Piece<Tx, C, true> px[KV];
  Piece<To, C, true> pz[KV], py[KV];
  auto load = [&](long r) {
#pragma unroll
    for (int k = 0; k < KV; ++k) {
      px[k].load(x + r * a.x_row + c[k], C);
      if (z) pz[k].load(z + r * a.z_row + c[k], C);
      if constexpr (BWD) py[k].load(dy + r * a.C + c[k], C);
    }
  };
  if (!LEAN && chunk < a.rows) load(chunk);
  for (long r = chunk; r < a.rows; r += tm.chunks) {
    float v[KV][C], zv[KV][C], gv[KV][C], sum = 0.f, sq = 0.f;
    if constexpr (LEAN) load(r);
#pragma unroll
    for (int k = 0; k < KV; ++k)
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const bool on = nv[k] > 0;
        v[k][i] = on ? px[k].get(i) : 0.f;
        zv[k][i] = on && z ? pz[k].get(i) : 0.f;
        if constexpr (BWD) gv[k][i] = on ? py[k].get(i) : 0.f;
        sum += v[k][i];
      }
    if (!LEAN && r + tm.chunks < a.rows) load(r + tm.chunks);
    const float mean = gn_sum<TEAM>(sum, team, lds) * inv;
#pragma unroll
    for (int k = 0; k < KV; ++k)
#pragma unroll
      for (int i = 0; i < C; ++i) {
        v[k][i] = nv[k] > 0 ? v[k][i] - mean : 0.f;
        sq = fmaf(v[k][i], v[k][i], sq);
      }
    const float rstd = rsqrtf(gn_sum<TEAM>(sq, team, lds) * inv + a.eps);
    if constexpr (!BWD) {
#pragma unroll
      for (int k = 0; k < KV; ++k) {
        float y[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const float n = fmaf(v[k][i] * rstd, w[k][i], b[k][i]);
          y[i] = z ? n * act_of(a.act, zv[k][i]) : act_of(a.act, n);
        }
        store_piece<To, C, true>(static_cast<To*>(a.y) + r * a.C + c[k], y, nv[k]);
      }
    } else {
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int k = 0; k < KV; ++k) {
        float dz[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const float xh = v[k][i] * rstd, n = fmaf(xh, w[k][i], b[k][i]);
          float y;
          const float sl = act_slope(a.act, z ? zv[k][i] : n, y);
          const float dn = gv[k][i] * (z ? y : sl);
          dz[i] = gv[k][i] * n * sl;
          if constexpr (LEAN) {
            kept[0][k][l] = fmaf(dn, xh, kept[0][k][l]);
            kept[1][k][l] += dn;
          } else {
            dw[k][i] = fmaf(dn, xh, dw[k][i]);
            db[k][i] += dn;
          }
          v[k][i] = xh;
          gv[k][i] = dn * w[k][i];
          s1 += gv[k][i];
          s2 = fmaf(gv[k][i], xh, s2);
        }
        if (z) store_piece<To, C, true>(static_cast<To*>(a.dz) + r * a.C + c[k], dz, nv[k]);
      }
      s1 = gn_sum<TEAM>(s1, team, lds) * inv;
      s2 = gn_sum<TEAM>(s2, team, lds) * inv;
#pragma unroll
      for (int k = 0; k < KV; ++k) {
        float dx[C];
#pragma unroll
        for (int i = 0; i < C; ++i) dx[i] = rstd * (gv[k][i] - s1 - v[k][i] * s2);
        store_piece<Tx, C, true>(static_cast<Tx*>(a.dx) + r * a.C + c[k], dx, nv[k]);
      }
    }
  }
  if constexpr (BWD) {
#pragma unroll
    for (int k = 0; k < KV; ++k)
#pragma unroll
      for (int i = 0; i < C; ++i)
        if (nv[k] > 0) {
          a.part[((long)chunk * 2 + 0) * a.C + c[k] + i] = LEAN ? kept[0][k][l] : dw[k][i];
          a.part[((long)chunk * 2 + 1) * a.C + c[k] + i] = LEAN ? kept[1][k][l] : db[k][i];
        }
  }
}

// Groups too wide for registers: a workgroup per (group, chunk of rows), which
// reads its rows again from the caches.
template <typename Tx, typename To, int C, bool BWD>
__global__ __launch_bounds__(GN_WIDE) void k_group_norm_wide(GroupNormArgs a, GnTeam tm) {
  __shared__ float lds[GN_WIDE / 64];
  const int m = a.C / a.G, g = blockIdx.x % a.G, chunk = blockIdx.x / a.G;
  const float inv = 1.f / m;
  const To *zt = static_cast<const To*>(a.z), *dyt = static_cast<const To*>(a.dy);
  const float *wt = a.w ? a.w + (long)g * m : nullptr, *bt = a.b ? a.b + (long)g * m : nullptr;
  float* pw = BWD ? a.part + (long)chunk * 2 * a.C + (long)g * m : nullptr;
  // fn(first channel) for every piece of the thread
  auto pieces = [&](auto fn) {
    for (int c = threadIdx.x * C; c < m; c += GN_WIDE * C) fn(c);
  };
  if constexpr (BWD) {
    pieces([&](int c) {
      for (int i = 0; i < C; ++i) pw[c + i] = pw[a.C + c + i] = 0.f;
    });
  }
  for (long r = chunk; r < a.rows; r += tm.chunks) {
    const Tx* x = static_cast<const Tx*>(a.x) + r * a.x_row + (long)g * m;
    const To* z = zt ? zt + r * a.z_row + (long)g * m : nullptr;
    float sum = 0.f, sq = 0.f;
    pieces([&](int c) {
      Piece<Tx, C, true> p;
      p.load(x + c, C);
#pragma unroll
      for (int i = 0; i < C; ++i) sum += p.get(i);
    });
    const float mean = block_sum<GN_WIDE>(sum, lds) * inv;
    pieces([&](int c) {
      Piece<Tx, C, true> p;
      p.load(x + c, C);
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const float d = p.get(i) - mean;
        sq = fmaf(d, d, sq);
      }
    });
    const float rstd = rsqrtf(block_sum<GN_WIDE>(sq, lds) * inv + a.eps);
    if constexpr (!BWD) {
      pieces([&](int c) {
        Piece<Tx, C, true> p;
        Piece<To, C, true> pz;
        p.load(x + c, C);
        if (z) pz.load(z + c, C);
        float y[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const int at = c + i;
          const float n = fmaf((p.get(i) - mean) * rstd, wt ? wt[at] : 1.f, bt ? bt[at] : 0.f);
          y[i] = z ? n * act_of(a.act, pz.get(i)) : act_of(a.act, n);
        }
        store_piece<To, C, true>(static_cast<To*>(a.y) + r * a.C + (long)g * m + c, y, C);
      });
    } else {
      const long row = r * a.C + (long)g * m;
      float s1 = 0.f, s2 = 0.f;
      // fn(i, xh, dn, dn w, dz) for every channel of a piece
      auto grad = [&](int c, auto fn) {
        Piece<Tx, C, true> p;
        Piece<To, C, true> pz, py;
        p.load(x + c, C);
        if (z) pz.load(z + c, C);
        py.load(dyt + row + c, C);
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const int at = c + i;
          const float wv = wt ? wt[at] : 1.f, xh = (p.get(i) - mean) * rstd;
          const float n = fmaf(xh, wv, bt ? bt[at] : 0.f), gv = py.get(i);
          float y;
          const float sl = act_slope(a.act, z ? pz.get(i) : n, y), dn = gv * (z ? y : sl);
          fn(i, xh, dn, dn * wv, gv * n * sl);
        }
      };
      pieces([&](int c) {
        grad(c, [&](int i, float xh, float dn, float gw, float) {
          s1 += gw;
          s2 = fmaf(gw, xh, s2);
          pw[c + i] = fmaf(dn, xh, pw[c + i]);
          pw[a.C + c + i] += dn;
        });
      });
      s1 = block_sum<GN_WIDE>(s1, lds) * inv;
      s2 = block_sum<GN_WIDE>(s2, lds) * inv;
      pieces([&](int c) {
        float dx[C], dz[C];
        grad(c, [&](int i, float xh, float, float gw, float d) {
          dx[i] = rstd * (gw - s1 - xh * s2);
          dz[i] = d;
        });
        if (z) store_piece<To, C, true>(static_cast<To*>(a.dz) + row + c, dz, C);
        store_piece<Tx, C, true>(static_cast<Tx*>(a.dx) + row + c, dx, C);
      });
    }
  }
}

// dweight and dbias: the chunks' partial sums, each of 16 waves every 16th in
// order, then the waves in order.
constexpr int GN_WAVES = 16;
__global__ __launch_bounds__(64 * GN_WAVES) void k_group_norm_dw(GroupNormArgs a) {
  __shared__ float part[GN_WAVES][64];
  const int lane = lane_id(), w = wave_id_s();
  const long n = 2L * a.C, e = (long)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (e < n) {
#pragma unroll 8
    for (int r = w; r < a.blocks; r += GN_WAVES) s += a.part[r * n + e];
  }
  part[w][lane] = s;
  __syncthreads();
  if (w == 0 && e < n) {
    for (int i = 1; i < GN_WAVES; ++i) s += part[i][lane];
    if (e < a.C) { if (a.dw) a.dw[e] = s; }
    else if (a.db) a.db[e - a.C] = s;
  }
}

// The team of a group of m channels, and how many teams walk the rows: 1,024 lanes
// per CU (bf16, 16,384 x 4,096 channels, groups of 128: 512 / 1,024 / 2,048 lanes
// forward 106 / 84 / 95 us, backward 164 / 155 / 166, whole calls with the sums).
constexpr long GN_LANES = 1024;
static GnTeam gn_team(const GroupNormArgs& a, int& kv) {
  const int m = a.C / a.G, pieces = (m + GN_C - 1) / GN_C;
  GnTeam t{};
  t.team = 1;
  while (t.team < 64 && t.team * 2 < pieces) t.team *= 2;
  if (pieces > 4 * 64) t.team = pieces > 4 * 256 ? 512 : 256;
  const int need = (pieces + t.team - 1) / t.team;
  kv = need <= 2 ? 2 : need <= 4 ? 4 : 0;
  if (!kv) t.team = GN_WIDE;
  const long lanes = (long)a.G * t.team;
  long chunks = 256L * GN_LANES / lanes;  // lanes per CU
  chunks = chunks < 1 ? 1 : chunks > a.rows ? a.rows : chunks;
  t.chunks = (int)chunks;
  return t;
}

int group_norm_bwd_blocks(const GroupNormArgs& a) {
  int kv;
  return a.rows > 0 ? gn_team(a, kv).chunks : 0;
}

template <typename Tx, typename To, bool BWD>
static hipError_t run_group_norm(const GroupNormArgs& a0) {
  GroupNormArgs a = a0;
  if (a.rows > 0) {
    int kv;
    const GnTeam t = gn_team(a, kv);
    a.blocks = t.chunks;
    auto ok = [&](const void* p, size_t eb, long row) {
      return !p || ((uintptr_t)p % (GN_C * eb) == 0 && row % GN_C == 0);
    };
    // pieces of four channels, or of one for other groups and for slices that are not
    // aligned to four (bf16, 16,384 x 4,096, groups of 128, whole calls: 84 / 106 us forward,
    // 155 / 207 backward; pieces of four loaded one by one 139 and 274)
    const bool vec = (a.C / a.G) % GN_C == 0 && ok(a.x, sizeof(Tx), a.x_row) && ok(a.z, sizeof(To), a.z_row) &&
                     ok(a.y, sizeof(To), a.C) && ok(a.dy, sizeof(To), a.C) && ok(a.dx, sizeof(Tx), a.C) &&
                     ok(a.dz, sizeof(To), a.C);
    const int th = t.team > 64 ? t.team : 256;
    const long grid = ((long)t.chunks * a.G * t.team + th - 1) / th;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
#define GN_LAUNCH(KV, TEAM)                                                                      \
  if (vec) k_group_norm<Tx, To, KV, GN_C, TEAM, BWD><<<(unsigned)grid, th, 0, a.stream>>>(a, t); \
  else k_group_norm<Tx, To, KV * GN_C, 1, TEAM, BWD><<<(unsigned)grid, th, 0, a.stream>>>(a, t);
    if (kv == 2 && t.team <= 64) { GN_LAUNCH(2, 0) }
    else if (kv == 4 && t.team <= 64) { GN_LAUNCH(4, 0) }
    else if (kv == 2) { GN_LAUNCH(2, 256) }
    else if (kv == 4 && t.team == 256) { GN_LAUNCH(4, 256) }
    else if (kv == 4) { GN_LAUNCH(4, 512) }
#undef GN_LAUNCH
    else if (vec) k_group_norm_wide<Tx, To, GN_C, BWD><<<(unsigned)grid, th, 0, a.stream>>>(a, t);
    else k_group_norm_wide<Tx, To, 1, BWD><<<(unsigned)grid, th, 0, a.stream>>>(a, t);
  }
  if (BWD && (a.dw || a.db))
    k_group_norm_dw<<<(unsigned)((2L * a.C + 63) / 64), 64 * GN_WAVES, 0, a.stream>>>(a);
  return hipGetLastError();
}

#define GN_DISPATCH(BWD, a)                                        \
  ((a).x_bf16   ? run_group_norm<bf16_t, bf16_t, BWD>(a)           \
   : (a).out_bf16 ? run_group_norm<float, bf16_t, BWD>(a) : run_group_norm<float, float, BWD>(a))

hipError_t launch_group_norm_fwd(const GroupNormArgs& a) { return GN_DISPATCH(false, a); }
hipError_t launch_group_norm_bwd(const GroupNormArgs& a) { return GN_DISPATCH(true, a); }

}  // namespace comba
