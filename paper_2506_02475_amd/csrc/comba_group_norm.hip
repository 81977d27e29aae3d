// Group norm per token, channels last: mean and variance over the m = C / G
// channels of a group of one token, then weight and bias, then an activation of
// the result, or a gate y = n act(z):
//
//   n = (x - mean) rstd w + b,   y = act(n)  |  n act(z).
//
// Bound by bytes: every value is read and written once.  A group's channels lie
// in the registers of a team of 1..64 lanes (a power of two) or of a workgroup of
// 256, KV pieces of four per lane, so that mean and variance are two passes over
// registers.  A team keeps its group and walks rows, with weight and bias
// (backward: and their gradients' sums) in registers.  Groups of more than 4,096
// channels read x again from the caches (k_group_norm_wide).
#include "comba_layer_device.hpp"
#include "comba_layer_launch.h"

namespace comba {

constexpr int GN_C = 4;  // channels of a piece

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

// Sum over a workgroup of 256, the same in every thread.
__device__ __forceinline__ float block_sum(float x, float* lds) {
  x = team_sum(x, 64);
  if (lane_id() == 0) lds[wave_id()] = x;
  __syncthreads();
  const float s = (lds[0] + lds[1]) + (lds[2] + lds[3]);
  __syncthreads();
  return s;
}

// The same over the team: a wave's lanes, or the workgroup.
template <bool BLOCK>
__device__ __forceinline__ float gn_sum(float x, int team, float* lds) {
  if constexpr (BLOCK) return block_sum(x, lds);
  return team_sum(x, team);
}

struct GnTeam {
  int team;    // lanes
  int chunks;  // row chunks: team (group, chunk) takes rows chunk, chunk + chunks, ..
};

template <typename Tx, typename To, int KV, bool VEC, bool BLOCK, bool BWD>
__global__ __launch_bounds__(256) void k_group_norm(GroupNormArgs a, GnTeam tm) {
  __shared__ float lds[4];
  const int m = a.C / a.G, team = tm.team;
  const long id = ((long)blockIdx.x * 256 + threadIdx.x) / team;
  const int l = threadIdx.x & (team - 1);
  const int g = id % a.G, chunk = id / a.G;
  if (chunk >= tm.chunks) return;  // whole teams
  int c[KV], nv[KV];
  float w[KV][GN_C], b[KV][GN_C], dw[KV][GN_C], db[KV][GN_C];
#pragma unroll
  for (int k = 0; k < KV; ++k) {
    const int at = (k * team + l) * GN_C;  // in the group
    nv[k] = max(0, min(GN_C, m - at));
    c[k] = g * m + (nv[k] > 0 ? at : 0);
#pragma unroll
    for (int i = 0; i < GN_C; ++i) {
      const bool on = i < nv[k];
      w[k][i] = on ? (a.w ? a.w[c[k] + i] : 1.f) : 0.f;
      b[k][i] = on && a.b ? a.b[c[k] + i] : 0.f;
      dw[k][i] = db[k][i] = 0.f;
    }
  }
  const float inv = 1.f / m;
  const Tx* x = static_cast<const Tx*>(a.x);
  const To *z = static_cast<const To*>(a.z), *dy = static_cast<const To*>(a.dy);
  Piece<Tx, GN_C, VEC> px[KV];
  Piece<To, GN_C, VEC> pz[KV], py[KV];
  auto load = [&](long r) {
#pragma unroll
    for (int k = 0; k < KV; ++k) {
      px[k].load(x + r * a.x_row + c[k], max(nv[k], 1));
      if (z) pz[k].load(z + r * a.z_row + c[k], max(nv[k], 1));
      if constexpr (BWD) py[k].load(dy + r * a.C + c[k], max(nv[k], 1));
    }
  };
  if (chunk < a.rows) load(chunk);
  for (long r = chunk; r < a.rows; r += tm.chunks) {
    float v[KV][GN_C], zv[KV][GN_C], gv[KV][GN_C], sum = 0.f, sq = 0.f;
#pragma unroll
    for (int k = 0; k < KV; ++k)
#pragma unroll
      for (int i = 0; i < GN_C; ++i) {
        const bool on = i < nv[k];
        v[k][i] = on ? px[k].get(i) : 0.f;
        zv[k][i] = on && z ? pz[k].get(i) : 0.f;
        if constexpr (BWD) gv[k][i] = on ? py[k].get(i) : 0.f;
        sum += v[k][i];
      }
    if (r + tm.chunks < a.rows) load(r + tm.chunks);
    const float mean = gn_sum<BLOCK>(sum, team, lds) * inv;
#pragma unroll
    for (int k = 0; k < KV; ++k)
#pragma unroll
      for (int i = 0; i < GN_C; ++i) {
        v[k][i] = i < nv[k] ? v[k][i] - mean : 0.f;
        sq = fmaf(v[k][i], v[k][i], sq);
      }
    const float rstd = rsqrtf(gn_sum<BLOCK>(sq, team, lds) * inv + a.eps);
    if constexpr (!BWD) {
#pragma unroll
      for (int k = 0; k < KV; ++k) {
        float y[GN_C];
#pragma unroll
        for (int i = 0; i < GN_C; ++i) {
          const float n = fmaf(v[k][i] * rstd, w[k][i], b[k][i]);
          y[i] = z ? n * act_of(a.act, zv[k][i]) : act_of(a.act, n);
        }
        store_piece<To, GN_C, VEC>(static_cast<To*>(a.y) + r * a.C + c[k], y, nv[k]);
      }
    } else {
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int k = 0; k < KV; ++k) {
        float dz[GN_C];
#pragma unroll
        for (int i = 0; i < GN_C; ++i) {
          const float xh = v[k][i] * rstd, n = fmaf(xh, w[k][i], b[k][i]);
          float y;
          const float sl = act_slope(a.act, z ? zv[k][i] : n, y);
          const float dn = gv[k][i] * (z ? y : sl);
          dz[i] = gv[k][i] * n * sl;
          dw[k][i] = fmaf(dn, xh, dw[k][i]);
          db[k][i] += dn;
          v[k][i] = xh;
          gv[k][i] = dn * w[k][i];
          s1 += gv[k][i];
          s2 = fmaf(gv[k][i], xh, s2);
        }
        if (z) store_piece<To, GN_C, VEC>(static_cast<To*>(a.dz) + r * a.C + c[k], dz, nv[k]);
      }
      s1 = gn_sum<BLOCK>(s1, team, lds) * inv;
      s2 = gn_sum<BLOCK>(s2, team, lds) * inv;
#pragma unroll
      for (int k = 0; k < KV; ++k) {
        float dx[GN_C];
#pragma unroll
        for (int i = 0; i < GN_C; ++i) dx[i] = rstd * (gv[k][i] - s1 - v[k][i] * s2);
        store_piece<Tx, GN_C, VEC>(static_cast<Tx*>(a.dx) + r * a.C + c[k], dx, nv[k]);
      }
    }
  }
  if constexpr (BWD) {
#pragma unroll
    for (int k = 0; k < KV; ++k)
#pragma unroll
      for (int i = 0; i < GN_C; ++i)
        if (i < nv[k]) {
          a.part[((long)chunk * 2 + 0) * a.C + c[k] + i] = dw[k][i];
          a.part[((long)chunk * 2 + 1) * a.C + c[k] + i] = db[k][i];
        }
  }
}

// Groups too wide for registers: a workgroup per (group, chunk of rows).
template <typename Tx, typename To, bool BWD>
__global__ __launch_bounds__(256) void k_group_norm_wide(GroupNormArgs a, GnTeam tm) {
  __shared__ float lds[4];
  const int m = a.C / a.G, g = blockIdx.x % a.G, chunk = blockIdx.x / a.G;
  const float inv = 1.f / m;
  const To *zt = static_cast<const To*>(a.z), *dyt = static_cast<const To*>(a.dy);
  float* pw = BWD ? a.part + (long)chunk * 2 * a.C + g * m : nullptr;
  if constexpr (BWD) {
    for (int c = threadIdx.x; c < m; c += 256) pw[c] = pw[a.C + c] = 0.f;
  }
  for (long r = chunk; r < a.rows; r += tm.chunks) {
    const Tx* x = static_cast<const Tx*>(a.x) + r * a.x_row + g * m;
    const To* z = zt ? zt + r * a.z_row + g * m : nullptr;
    float sum = 0.f, sq = 0.f;
    for (int c = threadIdx.x; c < m; c += 256) sum += to_f(x[c]);
    const float mean = block_sum(sum, lds) * inv;
    for (int c = threadIdx.x; c < m; c += 256) {
      const float d = to_f(x[c]) - mean;
      sq = fmaf(d, d, sq);
    }
    const float rstd = rsqrtf(block_sum(sq, lds) * inv + a.eps);
    auto norm = [&](int c, float& xh, float& wv) {
      wv = a.w ? a.w[g * m + c] : 1.f;
      xh = (to_f(x[c]) - mean) * rstd;
      return fmaf(xh, wv, a.b ? a.b[g * m + c] : 0.f);
    };
    if constexpr (!BWD) {
      To* y = static_cast<To*>(a.y) + r * a.C + g * m;
      for (int c = threadIdx.x; c < m; c += 256) {
        float xh, wv;
        const float n = norm(c, xh, wv);
        store_elem(y + c, z ? n * act_of(a.act, to_f(z[c])) : act_of(a.act, n));
      }
    } else {
      const To* dy = dyt + r * a.C + g * m;
      Tx* dx = static_cast<Tx*>(a.dx) + r * a.C + g * m;
      float s1 = 0.f, s2 = 0.f;
      auto grad = [&](int c, float& xh, float& dn, float& dz) {
        float wv, y;
        const float n = norm(c, xh, wv), gv = to_f(dy[c]);
        const float sl = act_slope(a.act, z ? to_f(z[c]) : n, y);
        dn = gv * (z ? y : sl);
        dz = gv * n * sl;
        return dn * wv;
      };
      for (int c = threadIdx.x; c < m; c += 256) {
        float xh, dn, dz;
        const float gw = grad(c, xh, dn, dz);
        s1 += gw;
        s2 = fmaf(gw, xh, s2);
        pw[c] = fmaf(dn, xh, pw[c]);
        pw[a.C + c] += dn;
      }
      s1 = block_sum(s1, lds) * inv;
      s2 = block_sum(s2, lds) * inv;
      for (int c = threadIdx.x; c < m; c += 256) {
        float xh, dn, dz;
        const float gw = grad(c, xh, dn, dz);
        if (z) store_elem(static_cast<To*>(a.dz) + r * a.C + g * m + c, dz);
        store_elem(dx + c, rstd * (gw - s1 - xh * s2));
      }
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
// forward 102 / 84 / 92 us, backward 149 / 149 / 154).
constexpr long GN_LANES = 1024;
static GnTeam gn_team(const GroupNormArgs& a, int& kv) {
  const int m = a.C / a.G, pieces = (m + GN_C - 1) / GN_C;
  GnTeam t{};
  t.team = 1;
  while (t.team < 64 && t.team * 2 < pieces) t.team *= 2;
  if (pieces > 4 * 64) t.team = 256;
  const int need = (pieces + t.team - 1) / t.team;
  kv = need <= 2 ? 2 : need <= 4 ? 4 : 0;
  const long lanes = (long)a.G * (kv ? t.team : 256);
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
    const bool vec = (a.C / a.G) % GN_C == 0 && ok(a.x, sizeof(Tx), a.x_row) && ok(a.z, sizeof(To), a.z_row) &&
                     ok(a.y, sizeof(To), a.C) && ok(a.dy, sizeof(To), a.C) && ok(a.dx, sizeof(Tx), a.C) &&
                     ok(a.dz, sizeof(To), a.C);
    const long threads = (long)t.chunks * a.G * (kv ? t.team : 256), grid = (threads + 255) / 256;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
#define GN_LAUNCH(KV, BLOCK)                                                                       \
  if (vec) k_group_norm<Tx, To, KV, true, BLOCK, BWD><<<(unsigned)grid, 256, 0, a.stream>>>(a, t); \
  else k_group_norm<Tx, To, KV, false, BLOCK, BWD><<<(unsigned)grid, 256, 0, a.stream>>>(a, t);
    if (kv == 2 && t.team < 256) { GN_LAUNCH(2, false) }
    else if (kv == 4 && t.team < 256) { GN_LAUNCH(4, false) }
    else if (kv == 2) { GN_LAUNCH(2, true) }
    else if (kv == 4) { GN_LAUNCH(4, true) }
    else k_group_norm_wide<Tx, To, BWD><<<(unsigned)grid, 256, 0, a.stream>>>(a, t);
#undef GN_LAUNCH
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
