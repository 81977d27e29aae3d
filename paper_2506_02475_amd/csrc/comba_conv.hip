// Short causal depthwise convolution with a history (the K - 1 inputs before a
// sequence's first token), bias and SiLU, its backward, and its single-token form:
//
//   u_t = bias + sum_j w_j xt_{t+j},   y_t = act(u_t),   xt = [h0; x].
//
// Streaming kernels, bound by bytes: a thread holds C consecutive channels and
// walks a run of tokens with the K - 1 previous rows in registers, so a row is
// read once but for the runs' first K - 1 rows.  4 x 4,096 tokens, 4,096 channels,
// 4 taps, bf16: forward 49 us (5.5 TB/s), backward 92 us (4.4 TB/s: the runs' own
// rows; 9% more is read again at their ends) and 6 for the sums.
#include "comba_layer_device.hpp"
#include "comba_layer_launch.h"

namespace comba {

constexpr int CONV_PF = 4;        // rows loaded ahead, together
constexpr int CONV_BWAVES = 4;    // runs of a workgroup of the backward

// Tokens per run: 32, or 16 or 8 where 32 would leave less than three waves a
// SIMD (a run reads K - 1 rows more than its own; the backward forms as many du
// more).  us by run 8 / 16 / 32 / 64, bf16: forward 16,384 tokens x 4,096 channels
// 54 / 50 / 49 / 51; 16,384 x 2,048: 29 / 26 / 26 / 27; 1,000 x 2,048: 5.3 / 5.9 / 7.8 /
// 12; backward 137 / 113 / 99 / 103; 72 / 54 / 46 / 46; 12 / 12 / 16 / 23.
static int conv_run(const ConvArgs& a, int C) {
  const long items = (long)a.Ttot * ((a.D + C - 1) / C);
  return items >= 32L * 192 * 1024 ? 32 : items >= 16L * 64 * 1024 ? 16 : 8;
}

// The non-empty sequence s = [sa, se) that holds token t (0 <= t < Ttot), inside
// the tokens whatever the offsets hold.
__device__ __forceinline__ void seq_of_token(const int32_t* __restrict__ cu, int N, int Tseq, int Ttot,
                                             int t, int& s, int& sa, int& se) {
  if (!cu) {
    s = t / Tseq;
    sa = s * Tseq;
    se = sa + Tseq;
    return;
  }
  int lo = 0, hi = N - 1;  // the last s with cu[s] <= t
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cu[mid] <= t) lo = mid; else hi = mid - 1;
  }
  s = lo;
  sa = min(max(cu[lo], 0), t);
  se = min(max(cu[lo + 1], t + 1), Ttot);
}

template <int K, int C>
__device__ __forceinline__ void load_taps(const float* __restrict__ w, int c, float (&wt)[K][C]) {
#pragma unroll
  for (int i = 0; i < C; ++i)
#pragma unroll
    for (int j = 0; j < K; ++j) wt[j][i] = w[(long)(c + i) * K + j];
}

// Row `pos` of sequence s (negative: its history) as floats.
template <typename Tin, int K, int C>
__device__ __forceinline__ void load_ext(const ConvArgs& a, int s, int sa, int pos, int c,
                                         float (&v)[C]) {
  Piece<Tin, C, true> p;
  if (pos >= 0) {
    p.load(static_cast<const Tin*>(a.x) + (long)(sa + pos) * a.x_row + c, C);
  } else if (a.h0) {
    p.load(static_cast<const Tin*>(a.h0) + ((long)s * (K - 1) + (K - 1) + pos) * a.D + c, C);
  } else {
    p.zero();
  }
#pragma unroll
  for (int i = 0; i < C; ++i) v[i] = p.get(i);
}

template <typename Tin, int K, int C>
__global__ __launch_bounds__(256) void k_conv_fwd(ConvArgs a) {
  const int pieces = a.D / C, nruns = (a.Ttot + a.run - 1) / a.run;
  const long e = (long)blockIdx.x * 256 + threadIdx.x;
  const long r = e / pieces;
  const int c = e % pieces * C;
  if (r >= nruns) {  // the final histories
    const long k = r - nruns;
    if (!a.ht || k >= (long)a.N * (K - 1)) return;
    const int s = k / (K - 1), j = k % (K - 1);
    int sa, se;
    seq_range(a.cu_seqlens, s, a.Tseq, a.Ttot, sa, se);
    float v[C];
    load_ext<Tin, K, C>(a, s, sa, se - sa - (K - 1) + j, c, v);
    store_piece<Tin, C, true>(static_cast<Tin*>(a.ht) + k * a.D + c, v, C);
    return;
  }
  const int t0 = r * a.run, t1 = min(t0 + a.run, a.Ttot);
  float wt[K][C], b[C], xw[K - 1][C];
  load_taps<K, C>(a.w, c, wt);
#pragma unroll
  for (int i = 0; i < C; ++i) b[i] = a.bias ? a.bias[c + i] : 0.f;
  const Tin* x = static_cast<const Tin*>(a.x) + c;
  Tin* y = static_cast<Tin*>(a.y) + c;
  int s, sa, se;
  seq_of_token(a.cu_seqlens, a.N, a.Tseq, a.Ttot, t0, s, sa, se);
#pragma unroll
  for (int m = 0; m < K - 1; ++m) load_ext<Tin, K, C>(a, s, sa, t0 - sa - (K - 1) + m, c, xw[m]);
  Piece<Tin, C, true> xr[CONV_PF];
#pragma unroll
  for (int k = 0; k < CONV_PF; ++k) xr[k].load(x + (long)min(t0 + k, t1 - 1) * a.x_row, C);
  for (int tb = t0; tb < t1; tb += CONV_PF) {
    Piece<Tin, C, true> xn[CONV_PF];
#pragma unroll
    for (int k = 0; k < CONV_PF; ++k) xn[k].load(x + (long)min(tb + CONV_PF + k, t1 - 1) * a.x_row, C);
    auto token = [&](int k) {
      const int t = tb + k;
      float o[C];
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const float xv = xr[k].get(i);
        float u = b[i];
#pragma unroll
        for (int m = 0; m < K - 1; ++m) u = fmaf(wt[m][i], xw[m][i], u);
        u = fmaf(wt[K - 1][i], xv, u);
        o[i] = a.silu ? u * sigmoid_acc(u) : u;
#pragma unroll
        for (int m = 0; m < K - 2; ++m) xw[m][i] = xw[m + 1][i];
        xw[K - 2][i] = xv;
      }
      store_piece<Tin, C, true>(y + (long)t * a.D, o, C);
    };
    if (tb + CONV_PF <= min(t1, se)) {  // inside one sequence: straight-line code
#pragma unroll
      for (int k = 0; k < CONV_PF; ++k) token(k);
    } else {
#pragma unroll
      for (int k = 0; k < CONV_PF; ++k) {
        const int t = tb + k;
        if (t < t1) {
          if (t >= se) {  // the next sequence starts with its own history
            seq_of_token(a.cu_seqlens, a.N, a.Tseq, a.Ttot, t, s, sa, se);
#pragma unroll
            for (int m = 0; m < K - 1; ++m) load_ext<Tin, K, C>(a, s, sa, m - (K - 1), c, xw[m]);
          }
          token(k);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < CONV_PF; ++k) xr[k] = xn[k];
  }
}

// One token per row; the state's rows move up by one.  A thread takes its
// channels of R rows, so that the taps, twice a row's bytes, are read once.  64
// rows of 4,096 channels: 3.2 us, less than the host takes for the call.
template <typename Tin, int K, int C, int R>
__global__ __launch_bounds__(256) void k_conv_step(ConvArgs a) {
  const int pieces = a.D / C;
  const long e = (long)blockIdx.x * 256 + threadIdx.x;
  const long row0 = e / pieces * R;
  if (row0 >= a.N) return;
  const int c = e % pieces * C;
  int slot[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const long row = min(row0 + r, (long)a.N - 1);
    slot[r] = a.slots ? a.slots[row] : (int)row;
  }
  Piece<Tin, C, true> p[R][K];
  Tin* st[R];
  bool on[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    on[r] = slot[r] >= 0 && slot[r] < a.num_slots;  // else padding
    st[r] = static_cast<Tin*>(a.state) + (long)(on[r] ? slot[r] : 0) * (K - 1) * a.D + c;
    if (a.num_slots > 0) {
#pragma unroll
      for (int j = 0; j < K - 1; ++j) p[r][j].load(st[r] + (long)j * a.D, C);
    }
    p[r][K - 1].load(static_cast<const Tin*>(a.x) + min(row0 + r, (long)a.N - 1) * a.x_row + c, C);
  }
  float wt[K][C], b[C];
  load_taps<K, C>(a.w, c, wt);
#pragma unroll
  for (int i = 0; i < C; ++i) b[i] = a.bias ? a.bias[c + i] : 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (row0 + r >= a.N) break;
    float o[C], v[K][C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float u = b[i];
#pragma unroll
      for (int j = 0; j < K; ++j) {
        v[j][i] = p[r][j].get(i);
        u = fmaf(wt[j][i], v[j][i], u);
      }
      o[i] = on[r] ? (a.silu ? u * sigmoid_acc(u) : u) : 0.f;
    }
    store_piece<Tin, C, true>(static_cast<Tin*>(a.y) + (row0 + r) * a.D + c, o, C);
    if (on[r]) {
#pragma unroll
      for (int j = 0; j < K - 1; ++j) store_piece<Tin, C, true>(st[r] + (long)j * a.D, v[j + 1], C);
    }
  }
}

// Backward.  du_t = dy_t act'(u_t) adds w_j du_t to row t - (K - 1) + j of the
// extended input; a run forms du for its own tokens and the K - 1 after them,
// and keeps the K rows still open in registers.  Rows before a sequence's first
// token are its history's; dht adds to the last K - 1 extended rows.  A run's dw
// and dbias are summed over the workgroup's runs in LDS.
template <typename Tin, int K, int C>
__global__ __launch_bounds__(64 * CONV_BWAVES) void k_conv_bwd(ConvArgs a) {
  __shared__ float part[CONV_BWAVES][K + 1][C][64];
  const int pieces = a.D / C, pgs = (pieces + 63) / 64;
  const int pg = blockIdx.x % pgs, rb = blockIdx.x / pgs;
  const int lane = lane_id(), w = wave_id_s();
  const int piece = pg * 64 + lane;
  const int c = min(piece, pieces - 1) * C, nv = piece < pieces ? C : 0;  // channels stored
  const int t0 = (rb * CONV_BWAVES + w) * a.run, t1 = min(t0 + a.run, a.Ttot);
  float dw[K][C], db[C];
#pragma unroll
  for (int i = 0; i < C; ++i) {
    db[i] = 0.f;
#pragma unroll
    for (int j = 0; j < K; ++j) dw[j][i] = 0.f;
  }
  if (t0 < a.Ttot) {
    float wt[K][C], b[C], xw[K - 1][C], acc[K][C];
    load_taps<K, C>(a.w, c, wt);
#pragma unroll
    for (int i = 0; i < C; ++i) b[i] = a.bias ? a.bias[c + i] : 0.f;
    int s, sa, se;
    seq_of_token(a.cu_seqlens, a.N, a.Tseq, a.Ttot, t0, s, sa, se);
    auto enter = [&](int t) {  // the window before token t of sequence s
#pragma unroll
      for (int m = 0; m < K - 1; ++m) load_ext<Tin, K, C>(a, s, sa, t - sa - (K - 1) + m, c, xw[m]);
#pragma unroll
      for (int m = 0; m < K; ++m)
#pragma unroll
        for (int i = 0; i < C; ++i) acc[m][i] = 0.f;
    };
    // row r of the tokens (before sa: history) is complete
    auto put = [&](int r, const float (&v)[C]) {
      const int ext = r - sa + (K - 1), tail = ext - (se - sa);  // tail >= 0: row of ht
      const bool tok = r >= sa;
      if (tok ? (r < t0 || r >= t1) : (!a.dh0 || sa < t0 || sa >= t1)) return;
      float o[C];
#pragma unroll
      for (int i = 0; i < C; ++i) o[i] = v[i];
      if (a.dht && tail >= 0) {
        Piece<Tin, C, true> p;
        p.load(static_cast<const Tin*>(a.dht) + ((long)s * (K - 1) + tail) * a.D + c, C);
#pragma unroll
        for (int i = 0; i < C; ++i) o[i] += p.get(i);
      }
      Tin* at = tok ? static_cast<Tin*>(a.dx) + (long)r * a.D + c
                    : static_cast<Tin*>(a.dh0) + ((long)s * (K - 1) + ext) * a.D + c;
      store_piece<Tin, C, true>(at, o, nv);
    };
    enter(t0);
    const Tin *x = static_cast<const Tin*>(a.x) + c, *dy = static_cast<const Tin*>(a.dy) + c;
    const int tstop = min(t1 + K - 1, a.Ttot);
    bool done = false;
    Piece<Tin, C, true> xb[CONV_PF], gb[CONV_PF], xn[CONV_PF], gn[CONV_PF];
    auto load = [&](int tb, Piece<Tin, C, true>(&xp)[CONV_PF], Piece<Tin, C, true>(&gp)[CONV_PF]) {
#pragma unroll
      for (int k = 0; k < CONV_PF; ++k) {
        const long row = min(tb + k, tstop - 1);
        xp[k].load(x + row * a.x_row, C);
        gp[k].load(dy + row * a.D, C);
      }
    };
    load(t0, xb, gb);
    for (int tb = t0; tb < tstop && !done; tb += CONV_PF) {
      load(tb + CONV_PF, xn, gn);  // in flight while this block is worked on
      // du of token tb + k, its part of the open rows and (mine) of dw and dbias;
      // row t - (K - 1) is then complete in acc[0]
      auto token = [&](int k, bool mine) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const float xv = xb[k].get(i);
          float u = b[i];
#pragma unroll
          for (int m = 0; m < K - 1; ++m) u = fmaf(wt[m][i], xw[m][i], u);
          u = fmaf(wt[K - 1][i], xv, u);
          float du = gb[k].get(i);
          if (a.silu) {
            const float sg = sigmoid_acc(u);
            du *= sg * fmaf(u, 1.f - sg, 1.f);
          }
#pragma unroll
          for (int j = 0; j < K; ++j) acc[j][i] = fmaf(wt[j][i], du, acc[j][i]);
          if (mine) {
#pragma unroll
            for (int j = 0; j < K - 1; ++j) dw[j][i] = fmaf(du, xw[j][i], dw[j][i]);
            dw[K - 1][i] = fmaf(du, xv, dw[K - 1][i]);
            db[i] += du;
          }
#pragma unroll
          for (int m = 0; m < K - 2; ++m) xw[m][i] = xw[m + 1][i];
          xw[K - 2][i] = xv;
        }
      };
      auto next_row = [&]() {
#pragma unroll
        for (int i = 0; i < C; ++i) {
#pragma unroll
          for (int m = 0; m < K - 1; ++m) acc[m][i] = acc[m + 1][i];
          acc[K - 1][i] = 0.f;
        }
      };
      if (tb - (K - 1) >= max(t0, sa) && tb + CONV_PF <= min(t1, se)) {
        // the block and the rows it completes are this run's, inside one sequence
#pragma unroll
        for (int k = 0; k < CONV_PF; ++k) {
          token(k, true);
          store_piece<Tin, C, true>(static_cast<Tin*>(a.dx) + (long)(tb + k - (K - 1)) * a.D + c, acc[0], nv);
          next_row();
        }
      } else {
#pragma unroll
        for (int k = 0; k < CONV_PF; ++k) {
          const int t = tb + k;
          if (t >= tstop || done) continue;
          if (t >= se) {
#pragma unroll
            for (int m = 0; m < K - 1; ++m) put(t - (K - 1) + m, acc[m]);
            if (t >= t1) {
              done = true;
              continue;
            }
            seq_of_token(a.cu_seqlens, a.N, a.Tseq, a.Ttot, t, s, sa, se);
            enter(t);
          }
          token(k, t < t1);
          put(t - (K - 1), acc[0]);
          next_row();
        }
      }
#pragma unroll
      for (int k = 0; k < CONV_PF; ++k) {
        xb[k] = xn[k];
        gb[k] = gn[k];
      }
    }
    if (!done) {  // the tokens end here, or the walk stopped inside a sequence past t1
#pragma unroll
      for (int m = 0; m < K - 1; ++m) put(tstop - (K - 1) + m, acc[m]);
    }
  }
#pragma unroll
  for (int i = 0; i < C; ++i) {
#pragma unroll
    for (int j = 0; j < K; ++j) part[w][j][i][lane] = dw[j][i];
    part[w][K][i][lane] = db[i];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < (K + 1) * 64 * C; e += 64 * CONV_BWAVES) {
    const int j = e / (64 * C), ch = e % (64 * C), l = ch / C, i = ch % C;
    float v = part[0][j][i][l];
#pragma unroll
    for (int m = 1; m < CONV_BWAVES; ++m) v += part[m][j][i][l];
    const int cc = pg * 64 * C + ch;
    if (cc < a.D) a.part[((long)rb * (K + 1) + j) * a.D + cc] = v;
  }
}

// dw and dbias: the workgroups' partial sums in order, split over 16 groups of
// threads that are added in order; and the histories' gradients of empty sequences.
constexpr int CONV_DCOLS = 16, CONV_DGROUPS = 16;
template <typename Tin, int K>
__global__ __launch_bounds__(256) void k_conv_dw(ConvArgs a) {
  __shared__ float part[CONV_DGROUPS][CONV_DCOLS];
  const long n = (long)(K + 1) * a.D;
  const int nb = (n + CONV_DCOLS - 1) / CONV_DCOLS;
  if ((int)blockIdx.x >= nb) {  // one block per sequence
    const int s = blockIdx.x - nb;
    int sa, se;
    seq_range(a.cu_seqlens, s, a.Tseq, a.Ttot, sa, se);
    if (se > sa) return;
    for (int e = threadIdx.x; e < (K - 1) * a.D; e += 256) {
      const long at = (long)s * (K - 1) * a.D + e;
      static_cast<Tin*>(a.dh0)[at] = a.dht ? static_cast<const Tin*>(a.dht)[at] : Tin(0);
    }
    return;
  }
  const int col = threadIdx.x % CONV_DCOLS, grp = threadIdx.x / CONV_DCOLS;
  const long e = (long)blockIdx.x * CONV_DCOLS + col;
  float s = 0.f;
  if (e < n)
    for (int r = grp; r < a.nruns; r += CONV_DGROUPS) s += a.part[r * n + e];
  part[grp][col] = s;
  __syncthreads();
  if (grp == 0 && e < n) {
    for (int i = 1; i < CONV_DGROUPS; ++i) s += part[i][col];
    const int j = e / a.D;
    const long c = e % a.D;
    if (j < K) a.dw[c * K + j] = s;
    else if (a.dbias) a.dbias[c] = s;
  }
}

// Whether the width and the alignment of every tensor allow C channels a thread, as
// one load or store; else it takes two or one (the step: one).  Forward, us with two /
// one: bf16 16,384 x 4,094 and 4,095 54 / 66; eight channels loaded one by one
// would take 137.
static bool conv_fits(const ConvArgs& a, int C) {
  const long m = C * (a.bf16 ? 2 : 4);
  auto ok = [&](const void* p) { return !p || (uintptr_t)p % m == 0; };
  return a.D % C == 0 && a.x_row % C == 0 && ok(a.x) && ok(a.h0) && ok(a.y) && ok(a.ht) && ok(a.state) &&
         ok(a.dy) && ok(a.dht) && ok(a.dx) && ok(a.dh0);
}

// Channels of a thread of the backward: two give twice the waves, four read and
// write wider, from 64 MiB of x on.  us, two / four channels, with the sums: bf16
// 300 tokens x 256 channels 9.4 / 11.9; 1,000 x 2,048 11.8 / 13.2; 16,384 x 2,048 45.9 /
// 49.5; 16,384 x 4,096 105 / 105; 16,384 x 5,000 142 / 134; fp32 1,000 x 2,048 12.3 / 14.3;
// 16,384 x 2,048 90.3 / 88.8.  (Eight leave too few waves: 133 at 16,384 x 4,096.)
static int conv_bc(const ConvArgs& a) {
  return (long)a.Ttot * a.D * (a.bf16 ? 2 : 4) <= 64L << 20 ? 2 : 4;
}
// (From the shape alone: the workspace is sized before there are tensors.)
static int conv_bwd_run(const ConvArgs& a) { return conv_run(a, conv_bc(a)); }
int conv_bwd_runs(const ConvArgs& a) {
  const int tokens = conv_bwd_run(a) * CONV_BWAVES;
  return (a.Ttot + tokens - 1) / tokens;
}

template <typename Tin, int K, int C>
static hipError_t conv_fwd_main(ConvArgs a) {
  a.run = conv_run(a, C);
  const long items = ((long)(a.Ttot + a.run - 1) / a.run + (a.ht ? (long)a.N * (K - 1) : 0)) * (a.D / C);
  const long grid = (items + 255) / 256;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (grid == 0) return hipSuccess;
  k_conv_fwd<Tin, K, C><<<(unsigned)grid, 256, 0, a.stream>>>(a);
  return hipGetLastError();
}
template <typename Tin, int K>
static hipError_t run_conv_fwd(const ConvArgs& a) {
  // two channels, in fp32 four where they fit (bf16, us with 8 / 4 / 2: 16,384 x 4,096 52.8 /
  // 52.8 / 48.5; 16,384 x 2,048 30.2 / 26.8 / 25.8; 1,000 x 2,048 7.5 / 5.8 / 5.3; fp32 with 4 / 2:
  // 16,384 x 4,096 108.7 / 111.7; 16,384 x 2,048 44.6 / 48.1)
  if constexpr (sizeof(Tin) == 4) {
    if (conv_fits(a, 4)) return conv_fwd_main<Tin, K, 4>(a);
  }
  return conv_fits(a, 2) ? conv_fwd_main<Tin, K, 2>(a) : conv_fwd_main<Tin, K, 1>(a);
}
template <typename Tin, int K, int C, int R>
static hipError_t conv_step_main(const ConvArgs& a) {
  const long grid = ((long)((a.N + R - 1) / R) * (a.D / C) + 255) / 256;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  k_conv_step<Tin, K, C, R><<<(unsigned)grid, 256, 0, a.stream>>>(a);
  return hipGetLastError();
}
template <typename Tin, int K, int R>
static hipError_t conv_step_rows(const ConvArgs& a) {
  constexpr int C = 8 / (int)sizeof(Tin);
  return conv_fits(a, C) ? conv_step_main<Tin, K, C, R>(a) : conv_step_main<Tin, K, 1, R>(a);
}
template <typename Tin, int K>
static hipError_t run_conv_step(const ConvArgs& a) {
  // four rows a thread where that leaves two workgroups per CU (4,096 channels, us
  // with one / four rows: 128 rows 3.9 / 4.9; 256 5.5 / 5.5; 512 8.8 / 7.8; 1,024 15.2 / 11.7)
  return (long)a.N * a.D * (int)sizeof(Tin) >= 4L * 512 * 256 * 8 ? conv_step_rows<Tin, K, 4>(a)
                                                                   : conv_step_rows<Tin, K, 1>(a);
}
template <typename Tin, int K, int C>
static hipError_t conv_bwd_main(const ConvArgs& a) {
  const long pgs = (a.D / C + 63) / 64, grid = pgs * a.nruns;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (grid > 0) k_conv_bwd<Tin, K, C><<<(unsigned)grid, 64 * CONV_BWAVES, 0, a.stream>>>(a);
  return hipSuccess;
}
template <typename Tin, int K>
static hipError_t run_conv_bwd(const ConvArgs& a0) {
  ConvArgs a = a0;
  a.run = conv_bwd_run(a);
  a.nruns = conv_bwd_runs(a);
  const hipError_t st = conv_bc(a) == 4 && conv_fits(a, 4) ? conv_bwd_main<Tin, K, 4>(a)
                        : conv_fits(a, 2) ? conv_bwd_main<Tin, K, 2>(a) : conv_bwd_main<Tin, K, 1>(a);
  if (st != hipSuccess) return st;
  const long nb = ((long)(K + 1) * a.D + CONV_DCOLS - 1) / CONV_DCOLS + (a.dh0 ? a.N : 0);
  k_conv_dw<Tin, K><<<(unsigned)nb, 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

#define CONV_DISPATCH(fn, a)                                             \
  ((a).K == 2   ? ((a).bf16 ? fn<bf16_t, 2>(a) : fn<float, 2>(a))        \
   : (a).K == 3 ? ((a).bf16 ? fn<bf16_t, 3>(a) : fn<float, 3>(a))        \
   : (a).K == 4 ? ((a).bf16 ? fn<bf16_t, 4>(a) : fn<float, 4>(a)) : hipErrorInvalidValue)

hipError_t launch_conv_fwd(const ConvArgs& a) { return CONV_DISPATCH(run_conv_fwd, a); }
hipError_t launch_conv_step(const ConvArgs& a) { return a.N == 0 ? hipSuccess : CONV_DISPATCH(run_conv_step, a); }
hipError_t launch_conv_bwd(const ConvArgs& a) { return CONV_DISPATCH(run_conv_bwd, a); }

}  // namespace comba
