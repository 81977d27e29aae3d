// Internal interface between the host API (comba_layer_api.cpp) and the kernels
// of the layer's operators.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "comba_layer.h"

namespace comba {

struct ConvArgs {
  bool bf16, silu;
  int D, K, N, Tseq, Ttot;
  int run;     // tokens per run (set by the launcher)
  int nruns;   // backward: runs that leave a partial sum
  const int32_t* cu_seqlens;
  long x_row;
  const void *x, *h0;
  const float *w, *bias;
  void *y, *ht;
  // step
  void* state;
  const int32_t* slots;
  int num_slots;
  // backward
  const void *dy, *dht;
  void *dx, *dh0;
  float *dw, *dbias;
  float* part;  // [runs][K + 1][D] partial sums of dw and dbias
  hipStream_t stream;
};
// Runs of the backward, which size its workspace.
int conv_bwd_runs(const ConvArgs& a);
hipError_t launch_conv_fwd(const ConvArgs& a);
hipError_t launch_conv_bwd(const ConvArgs& a);
hipError_t launch_conv_step(const ConvArgs& a);

// Tokens between the states that the saving forward keeps for the backward, one
// tile of the backward (8 states per channel: the LDS of twelve waves would not fit).
constexpr int select_ck(int N) { return N == 8 ? 32 : 48; }
// A segment's length is a multiple of every kernel's tile.
constexpr int select_tile(int N) { return N == 8 ? 64 : 96; }

struct SelectArgs {
  bool bf16, softplus;
  int D, N, G, S, Tseq, Ttot;  // S sequences
  const int32_t* cu_seqlens;
  const int32_t* cu_host;  // the host's copy, or NULL (host code only)
  long longest;  // tokens of the longest sequence (packed without host offsets: 0)
  long u_row, delta_row, z_row, b_row, c_row;
  const void *u, *delta, *Bm, *Cm, *z;
  const float *A, *Dskip, *bias, *h0;
  void* y;
  float* ht;
  // states at every select_ck(N)-th token of each sequence: written (or NULL), read
  float* ck;
  const float* kept;
  // step
  float* state;
  const int32_t* slots;
  int num_slots;
  // backward
  const void* dy;
  const float* dht;
  void *du, *ddelta, *dz, *dB, *dC;
  float *dA, *dD, *dbias, *dh0;
  int nblk;      // channel blocks per group
  // sequences of more than `segmin` tokens cut into up to `segs` segments of
  // `seglen` tokens; a work row is a segment or a whole sequence: each segment's end
  // from zero and the sum of its steps
  int segs, seglen, segmin;
  float* segF;   // [work row][D][N]
  float* segdt;  // [work row][D]
  float* bcp;    // [channel block][token][2 N] partial dB, dC of one block's channels
  float* dap;    // [work row][D][N + 2] partial dA, dD, dbias
  hipStream_t stream;
};
// The work rows in the order of their workgroups.  Packed sequences with host
// offsets: rows at[i] .. at[i + 1] - 1 are the segments of sequence seq[i], the
// longest work first; the sequences not listed follow whole, in their own order.
constexpr int SEL_LIST = 32;
struct SelectRows {
  int rows, n;
  int32_t seq[SEL_LIST];
  int16_t at[SEL_LIST + 1];  // up to 32 segments each
};
// Channels of one workgroup of the backward, and its blocks per group.
constexpr int select_block_channels(int N) { return 512 / N; }
hipError_t launch_select_fwd(const SelectArgs& a, const SelectRows& q);
hipError_t launch_select_bwd(const SelectArgs& a, const SelectRows& q);
hipError_t launch_select_step(const SelectArgs& a);

struct GroupNormArgs {
  bool x_bf16, out_bf16;
  comba_activation act;
  long rows;
  int C, G;
  float eps;
  long x_row, z_row;
  const void *x, *z;
  const float *w, *b;
  void* y;
  const void* dy;
  void *dx, *dz;
  float *dw, *db;
  float* part;  // [blocks][2][C] partial sums of dw and db
  int blocks;
  hipStream_t stream;
};
// Workgroups of the backward over the rows, which size its workspace.
int group_norm_bwd_blocks(const GroupNormArgs& a);
hipError_t launch_group_norm_fwd(const GroupNormArgs& a);
hipError_t launch_group_norm_bwd(const GroupNormArgs& a);

}  // namespace comba
